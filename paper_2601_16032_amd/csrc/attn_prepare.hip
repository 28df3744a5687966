// attn_qkv_prepare: norms of queries and keys per head, position rotation, rows to where the attention reads them.
//
//   y = x * rsqrt(mean(x^2) + eps) * w,   (a, b) -> (a cos t - b sin t, a sin t + b cos t),   t = position * frequency[i]
//
// Bound by memory: a row of d elements is read once and written once (keys and values twice where both a tensor and the cache take
// them), at some 12 flops per element.  A row is held by d/8 lanes, eight elements each; a wavefront takes 4 (d = 128) or 8 rows
// of one token at a time, so that the angles, the same for all heads, are made once per token, one by each
// lane, which then takes the four it turns its four pairs of elements by from other lanes.  With pairs (i, i + rotated/2) a lane holds
// elements 4j.. and rotated/2 + 4j.., two pieces of 8 bytes, and no element changes lanes; with pairs (2i, 2i + 1) one piece of 16 bytes.
// Rows are stored non-temporally (2048 tokens of 48 heads 22.8 -> 14.8 us) and loaded a trip ahead.  32 + 2 x 8 heads x 16384 into the cache, 403 MB:
// 77 us, 5.2 TB/s (calls captured into a graph, inputs changing; the same bytes copied non-temporally 64 us, 6.3 TB/s).  Angles: position * frequency / 2 pi in 64 bits, less its nearest
// whole number; in 32 bits it would be off by 0.06 of a radian at position 10^6.  Sums, norms and turns are in 32 bits, and there is one
// rounding, to the type of the rows.
namespace sawattn {

constexpr int kPrepareThreads = 256;

struct Rows {
    char* data;
    long long sequence, token, head;      // strides in bytes
};

struct PrepareParams {
    Rows q, k, v, q_out, k_out, v_out;      // outputs with data NULL are not wanted
    char* cache_k;                          // NULL: no cache
    char* cache_v;
    long long k_page, k_head, k_row, v_page, v_head, v_row;      // bytes
    long long slots_end;
    int shift;
    const long long* slots;
    const int* positions;
    const float* q_weight;
    const float* k_weight;
    const double* frequencies;
    float eps;
    int rotated, tokens, N, H, KH, trips, chunks;      // a wavefront takes a token's rows in `trips` trips, `chunks` wavefronts take all
};

// x added up over the aligned group of LANES (8 or 16) lanes, in every lane.
template <int LANES>
__device__ __forceinline__ float group_sum(float x) {
    auto moved = [](float y, auto control) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, y), decltype(control)::value, 0xf, 0xf, true));
    };
    x += moved(x, std::integral_constant<int, 0xb1>{});       // neighbours, quad_perm [1,0,3,2]
    x += moved(x, std::integral_constant<int, 0x4e>{});       // pairs, quad_perm [2,3,0,1]
    x += moved(x, std::integral_constant<int, 0x141>{});      // quads: every lane of one holds the same, so that a mirrored half row does
    if constexpr (LANES == 16) x += moved(x, std::integral_constant<int, 0x140>{});
    return x;
}

template <bool BF16>
__device__ __forceinline__ float widen(unsigned word, int half) {
    if constexpr (BF16) return __builtin_bit_cast(float, half ? word & 0xffff0000u : word << 16);
    else return (float)__builtin_bit_cast(h2, word)[half];
}

template <bool BF16>
__device__ __forceinline__ unsigned narrow(float a, float b) {
    if constexpr (BF16) {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(unsigned, b2{(__bf16)a, (__bf16)b});
    } else {
        return __builtin_bit_cast(unsigned, h2{(_Float16)a, (_Float16)b});
    }
}

// AHEAD: the rows of a trip are on their way while those before are worked on, the first while the angles are made.
template <int D, bool BF16, bool INTERLEAVED, bool AHEAD>
__global__ __launch_bounds__(kPrepareThreads) void qkv_prepare_kernel(PrepareParams p) {
    constexpr int kLanes = D / 8, kRows = 64 / kLanes;
    const int lane = threadIdx.x & 63, j = lane % kLanes, group = lane / kLanes;
    const int unit = __builtin_amdgcn_readfirstlane(blockIdx.x * (kPrepareThreads / 64) + (threadIdx.x >> 6));
    const int t = unit / p.chunks, chunk = unit - t * p.chunks;
    if (t >= p.tokens) return;
    const int position = p.positions[t];
    if (position < 0) return;
    const int b = t / p.N, n = t - b * p.N;

    const bool turns = j < p.rotated / 8;
    // the lane's eight elements, in bytes: two pieces of four, or (one behind the other) one of eight
    const int low = (INTERLEAVED || !turns) ? 16 * j : 8 * j;
    const int high = (INTERLEAVED || !turns) ? 16 * j + 8 : p.rotated + 8 * j;
    f4 wq[2], wk[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int at = (i ? high : low) / 2;
        wq[i] = p.q_weight ? *reinterpret_cast<const f4*>(p.q_weight + at) : f4{1.f, 1.f, 1.f, 1.f};
        wk[i] = p.k_weight ? *reinterpret_cast<const f4*>(p.k_weight + at) : f4{1.f, 1.f, 1.f, 1.f};
    }
    long long page = -1;
    int page_row = 0;
    if (p.cache_k) {
        const long long slot = p.slots[t];
        if (slot >= 0 && slot < p.slots_end) {
            page = slot >> p.shift;
            page_row = (int)(slot & ((1 << p.shift) - 1));
        }
    }
    auto start = [&](const Rows& rows) { return rows.data + b * rows.sequence + n * rows.token; };
    const char* const q = start(p.q);
    const char* const k = start(p.k);
    const char* const v = start(p.v);
    char* const q_out = start(p.q_out);
    char* const k_out = p.k_out.data ? start(p.k_out) : nullptr;
    char* const v_out = p.v_out.data ? start(p.v_out) : nullptr;
    char* const k_slot = page >= 0 ? p.cache_k + page * p.k_page + page_row * p.k_row : nullptr;
    char* const v_slot = page >= 0 ? p.cache_v + page * p.v_page + page_row * p.v_row : nullptr;

    const int rows = p.H + 2 * p.KH, row0 = chunk * p.trips * kRows + group;
    struct Row {
        bool is_q, is_v;
        int head;
    };
    auto row_of = [&](int row) {
        const bool is_q = row < p.H, is_v = row >= p.H + p.KH;
        return Row{is_q, is_v, is_q ? row : is_v ? row - p.H - p.KH : row - p.H};
    };
    auto fetch = [&](const Row& row, u2 (&to)[2]) {      // the lane's pieces of it
        const char* from = row.is_q ? q + row.head * p.q.head : row.is_v ? v + row.head * p.v.head : k + row.head * p.k.head;
        if constexpr (INTERLEAVED) {
            const u4 both = *reinterpret_cast<const u4*>(from + low);
            to[0] = u2{both[0], both[1]};
            to[1] = u2{both[2], both[3]};
        } else {
            to[0] = *reinterpret_cast<const u2*>(from + low);
            to[1] = *reinterpret_cast<const u2*>(from + high);
        }
    };
    u2 coming[2] = {};
    if (AHEAD && row0 < rows) fetch(row_of(row0), coming);
    // One pair of a cosine and a sine per lane, those of the token's pairs of elements (in both halves of the wavefront at d = 64); a lane then
    // fetches the four it turns by.  Four per lane of a row cost more code than the rest of the kernel.
    float cosine[4], sine[4];
    {
        const int pair = lane % (D / 2);
        double turn = pair < p.rotated / 2 ? (double)position * p.frequencies[pair] * 0.15915494309189533577 : 0.;      // 1 / (2 pi)
        turn -= __builtin_rint(turn);
        float c, s;
        sincospif(2.f * (float)turn, &s, &c);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cosine[i] = __shfl(c, 4 * j + i);
            sine[i] = __shfl(s, 4 * j + i);
        }
    }
    for (int trip = 0; trip < p.trips; ++trip) {
        const int row = row0 + trip * kRows;
        if (row >= rows) break;
        const auto [is_q, is_v, head] = row_of(row);
        u2 x[2];
        if constexpr (AHEAD) {
            x[0] = coming[0];
            x[1] = coming[1];
            if (trip + 1 < p.trips && row + kRows < rows) fetch(row_of(row + kRows), coming);
        } else {
            fetch(Row{is_q, is_v, head}, x);
        }
        if (!is_v) {
            float y[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = widen<BF16>(x[e / 4][e / 2 % 2], e % 2);
            if (is_q ? p.q_weight != nullptr : p.k_weight != nullptr) {
                float square = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) square += y[e] * y[e];
                const float norm = 1.f / sqrtf(group_sum<kLanes>(square) * (1.f / D) + p.eps);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] *= norm * (is_q ? wq[e / 4][e % 4] : wk[e / 4][e % 4]);
            }
            if (turns) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int ea = INTERLEAVED ? 2 * i : i, eb = INTERLEAVED ? 2 * i + 1 : i + 4;
                    const float a = y[ea], c = y[eb];
                    y[ea] = a * cosine[i] - c * sine[i];
                    y[eb] = a * sine[i] + c * cosine[i];
                }
            }
#pragma unroll
            for (int e = 0; e < 8; e += 2) x[e / 4][e / 2 % 2] = narrow<BF16>(y[e], y[e + 1]);
        }
        auto put = [&](char* to) {
            if constexpr (INTERLEAVED) {
                __builtin_nontemporal_store(u4{x[0][0], x[0][1], x[1][0], x[1][1]}, reinterpret_cast<u4*>(to + low));
            } else {
                __builtin_nontemporal_store(x[0], reinterpret_cast<u2*>(to + low));
                __builtin_nontemporal_store(x[1], reinterpret_cast<u2*>(to + high));
            }
        };
        if (is_q) {
            put(q_out + head * p.q_out.head);
        } else if (!is_v) {
            if (k_out) put(k_out + head * p.k_out.head);
            if (k_slot) put(k_slot + head * p.k_head);
        } else {
            if (v_out) put(v_out + head * p.v_out.head);
            if (v_slot) put(v_slot + head * p.v_head);
        }
    }
}

template <int D, bool BF16>
void launch_prepare(const PrepareParams& p, bool interleaved, int grid, hipStream_t stream) {
    // Loading ahead, where there is anything to load ahead: 8192 tokens of 48 heads 49 -> 44 us, 16384 85 -> 77, 4096 28 -> 24, 1024 8.2 -> 7.7; a single
    // token (one trip) would take 3.3 instead of 3.2.
    auto launch = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(grid), dim3(kPrepareThreads), 0, stream, p); };
    if (interleaved) p.trips > 1 ? launch(qkv_prepare_kernel<D, BF16, true, true>) : launch(qkv_prepare_kernel<D, BF16, true, false>);
    else p.trips > 1 ? launch(qkv_prepare_kernel<D, BF16, false, true>) : launch(qkv_prepare_kernel<D, BF16, false, false>);
}

}  // namespace sawattn

extern "C" int attn_qkv_prepare(const sawattn_qkv* rows, const sawattn_kv_cache* cache, const int64_t* slots, const int32_t* positions,
                                const float* q_weight, const float* k_weight, float eps, const double* frequencies, int rotated,
                                int interleaved, int B, int N, int H, int KH, int d, int dtype, void* hip_stream) {
    using namespace sawattn;
    if (B <= 0 || N <= 0 || H <= 0 || KH <= 0 || d <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "B, N, H, KH and d must be positive");
    if (d != 64 && d != 128) return fail(SAWATTN_ERR_UNSUPPORTED, "head dimension must be 64 or 128");
    if (dtype != SAWATTN_F16 && dtype != SAWATTN_BF16)
        return fail(SAWATTN_ERR_INVALID_ARG, "dtype must be SAWATTN_F16 or SAWATTN_BF16");
    if ((long long)B * N >= (1LL << 26) || H > (1 << 16) || KH > (1 << 16) || H + 2LL * KH > (1 << 16))
        return fail(SAWATTN_ERR_INVALID_ARG, "B*N must be below 2^26 and H + 2*KH at most 2^16");
    if (rotated < 0 || rotated > d || rotated % 8) return fail(SAWATTN_ERR_INVALID_ARG, "rotated must be a multiple of 8 from 0 to d");
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(SAWATTN_ERR_INVALID_ARG, "eps must be finite and not negative");
    if (!rows || !rows->q.data || !rows->k.data || !rows->v.data || !rows->q_out.data || !positions || (rotated && !frequencies))
        return fail(SAWATTN_ERR_INVALID_ARG, "q, k, v, q_out, positions and (with rotated > 0) frequencies must be non-null");
    if ((rows->k_out.data == nullptr) != (rows->v_out.data == nullptr)) return fail(SAWATTN_ERR_INVALID_ARG, "k_out and v_out must be given together");
    if ((cache == nullptr) != (slots == nullptr)) return fail(SAWATTN_ERR_INVALID_ARG, "cache and slots must be given together");
    if (((uintptr_t)q_weight | (uintptr_t)k_weight | (uintptr_t)frequencies) & 15u)
        return fail(SAWATTN_ERR_INVALID_ARG, "q_weight, k_weight and frequencies must be 16-byte aligned");
    if (((uintptr_t)positions & 3u) || ((uintptr_t)slots & 7u))
        return fail(SAWATTN_ERR_INVALID_ARG, "positions and slots must be aligned to their elements");
    PrepareParams p{};
    const struct { const sawattn_rows* from; Rows* to; int heads; } tensors[] = {
        {&rows->q, &p.q, H}, {&rows->k, &p.k, KH}, {&rows->v, &p.v, KH}, {&rows->q_out, &p.q_out, H}, {&rows->k_out, &p.k_out, KH}, {&rows->v_out, &p.v_out, KH}};
    for (int i = 0; i < 6; ++i) {
        const sawattn_rows* s = tensors[i].from;
        if (!s->data) continue;
        if ((uintptr_t)s->data & 15u) return fail(SAWATTN_ERR_INVALID_ARG, "rows must be 16-byte aligned");
        if (!good_stride(s->sequence, B) || !good_stride(s->token, N) || !good_stride(s->head, tensors[i].heads))
            return fail(SAWATTN_ERR_INVALID_ARG, "strides of rows must be multiples of 8, not negative");
        // rows written must be rows of their own
        if (i >= 3 && ((B > 1 && s->sequence < d) || (N > 1 && s->token < d) || (tensors[i].heads > 1 && s->head < d)))
            return fail(SAWATTN_ERR_INVALID_ARG, "strides of rows that are written must be at least d");
        *tensors[i].to = {static_cast<char*>(s->data), 2 * s->sequence, 2 * s->token, 2 * s->head};
    }
    if (cache) {
        const int rc = check_cache(cache, true);
        if (rc != SAWATTN_OK) return rc;
        if (cache->heads != KH || cache->d != d || cache->dtype != dtype)
            return fail(SAWATTN_ERR_INVALID_ARG, "the cache's heads, d and dtype must be those of K and V");
        for (const int64_t* s : {&cache->k_page, &cache->v_page})      // page, head and row strides lie one behind the other
            if ((cache->pages > 1 && s[0] < d) || (KH > 1 && s[1] < d) || s[2] < d)
                return fail(SAWATTN_ERR_INVALID_ARG, "strides of a cache that is written must be at least d");
        p.cache_k = static_cast<char*>(cache->k);
        p.cache_v = static_cast<char*>(cache->v);
        p.k_page = 2 * cache->k_page; p.k_head = 2 * cache->k_head; p.k_row = 2 * cache->k_row;
        p.v_page = 2 * cache->v_page; p.v_head = 2 * cache->v_head; p.v_row = 2 * cache->v_row;
        p.shift = page_shift(cache->page_size);
        p.slots_end = (long long)cache->pages << p.shift;
        p.slots = reinterpret_cast<const long long*>(slots);
    }
    p.positions = positions;
    p.q_weight = q_weight; p.k_weight = k_weight; p.frequencies = frequencies;
    p.eps = eps; p.rotated = rotated; p.tokens = B * N; p.N = N; p.H = H; p.KH = KH;
    // A wavefront takes all rows of a token, or, where that would make fewer than 4096 wavefronts, fewer of them, 4 (d = 128) or 8 at least.  Measured, 32 +
    // 2 x 8 heads of 128 into the cache, 2048, 4096 and 8192 wavefronts: 1024 tokens 8.7, 7.6, 7.8 us; 2048 tokens 13.8, 11.5, 12.3; 4096 tokens 24.2, 23.5, 25.0.
    const int heads = H + 2 * KH, at_once = 64 / (d / 8), all = (heads + at_once - 1) / at_once;
    const int wanted = (int)std::min<long long>(all, (4096 + p.tokens - 1) / p.tokens);
    p.trips = (all + wanted - 1) / wanted;
    p.chunks = (all + p.trips - 1) / p.trips;
    const long long waves = (long long)p.tokens * p.chunks;      // (below 2^26: 4096 tokens and more have one each, fewer at most 2^14)
    const int grid = (int)((waves + kPrepareThreads / 64 - 1) / (kPrepareThreads / 64));
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const bool bf = dtype == SAWATTN_BF16;
    if (d == 128) bf ? launch_prepare<128, true>(p, interleaved != 0, grid, stream) : launch_prepare<128, false>(p, interleaved != 0, grid, stream);
    else bf ? launch_prepare<64, true>(p, interleaved != 0, grid, stream) : launch_prepare<64, false>(p, interleaved != 0, grid, stream);
    return launched("attn_qkv_prepare");
}
