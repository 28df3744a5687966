// attn_decode: attention of one new token per request over a paged key-value cache.
//
//   s_j = scale q . k_j,  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)   over the visible rows j of a request
//
// Bound by memory: every key and value is read once, for 4 d flops per query head that shares it.  A unit is a request, a key/value
// head and up to 16 of its query heads; its rows are cut into tiles of 32.  The tiles of all units, one behind the other, are dealt
// out evenly: workgroup w of G takes `share` of them from w * share on, whatever the lengths are, so that one long request and many
// short ones load the chip alike and the launch needs to know no length on the host.  Where a unit is spread over workgroups each leaves
// (m, sum, O) of its part in the workspace, and a second kernel joins them.  A workgroup ends at most two units unfinished, its first and
// its last, so the workspace has two places per workgroup.
//
// Within a workgroup the four wavefronts take every fourth tile, each with its own running maximum and sum, and are added up in LDS at the
// unit's end.  Products run on 16x16x32 MFMAs, transposed: S^T = K Q^T, O^T = V^T P^T with the 16 columns the query heads (columns without
// one are computed and dropped: the matrix cores idle anyway).  K goes from memory straight into A operands.  In the result a lane holds
// eight scores of one head: four rows of S^T in each of two MFMAs.  With row i + 4 g + 16 mt of the two standing for key 8 g + 4 mt + i,
// these are keys 8 g .. 8 g + 7, which is what the lane has to hold of P^T as B operand of the second product: probabilities stay where
// they are.  V comes as eight rows of a lane group's keys, 16 bytes (8 bytes at d = 64) of each per lane; pairs of rows are interleaved in
// registers (v_perm) into A operands whose MFMA j has the elements j, j + 8, ... of V: neither K nor V passes LDS.
//
// The probabilities enter the second product as the sum of two 16-bit numbers, so that they are not rounded: the matrix cores have time
// for both.  Binary16 ones are scaled by 2^12 for the sake of small ones.
namespace sawattn {

constexpr int kDecodeThreads = 256, kDecodeWaves = kDecodeThreads / 64;
constexpr int kDecodeTile = 32;           // keys of a tile
constexpr int kDecodeHeads = 16;          // query heads of a unit
constexpr int kDecodeGrid = 1024;         // workgroups at most
constexpr int kDecodeLeast = 8;           // tiles of a workgroup at least

struct DecodeParams {
    const char* Q;
    char* O;
    long long q_request, q_head, o_request, o_head;      // bytes
    const char* K;
    const char* V;
    long long k_page, k_head, k_row, v_page, v_head, v_row;      // bytes
    const int* table;
    long long table_stride;
    const int* lengths;
    float* parts;        // workspace: [2 * grid][heads_kept][D] of O
    f2* part_sums;       // [2 * grid][heads_kept] of (maximum, sum)
    float c;             // scale * log2(e)
    int o_dtype, R, capacity, window, pages, shift;
    int group;           // query heads per key/value head
    int head_groups;     // units per request and key/value head
    int units;           // per request
    int heads_kept;      // of a unit: min(group, 16)
};

struct DecodeRequest {
    int length, low, first, tiles;      // visible rows low .. length - 1, in tiles from `first` on
    __device__ __forceinline__ DecodeRequest(const DecodeParams& p, int given) {
        length = min(max(given, 0), p.capacity);
        low = p.window ? max(length - p.window, 0) : 0;
        first = low / kDecodeTile;
        tiles = length ? (length - 1) / kDecodeTile - first + 1 : 0;
    }
};

__device__ __forceinline__ long long divide(long long a, long long b) {      // of numbers that are not negative, mostly of few bits
    if (((a | b) >> 31) == 0) return (unsigned)a / (unsigned)b;
    return a / b;
}

// How the tiles are dealt out: the same in both kernels, from the lengths alone.  Every wavefront works it out for itself.
struct DecodeShares {
    long long share;
    // ALL: the sum over all requests gives the share; tiles of the requests before request `of` (if not negative) in `before`
    long long before;
    __device__ __forceinline__ DecodeShares(const DecodeParams& p, int lane, int grid, int of) {
        long long all = 0, ahead = 0;
        for (int r = lane; r < p.R; r += 64) {
            const int n = DecodeRequest(p, p.lengths[r]).tiles;
            all += n;
            if (r < of) ahead += n;
        }
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            all += __shfl_xor(all, step);
            ahead += __shfl_xor(ahead, step);
        }
        share = divide(all * p.units + grid - 1, grid);
        share = max((long long)kDecodeLeast, (share + kDecodeWaves - 1) / kDecodeWaves * kDecodeWaves);
        before = ahead;
        total = all * p.units;
    }
    long long total;
};

template <bool BF16>
__device__ __forceinline__ f4 decode_mfma(u4 a, u4 b, f4 c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// What a unit's tiles need of its request and head.
struct DecodeUnit {
    const char* K;
    const char* V;
    const int* pages;
    int low, length;
};

template <int D>
struct DecodeTile {
    u4 k[2][D / 32];            // A operands: [rows of S^T][32 elements]
    unsigned v[8][D / 32];      // eight rows of V, D / 32 words of each
    bool bad_k, bad_v;

    __device__ __forceinline__ void load(const DecodeParams& p, const DecodeUnit& u, int tile, int lane) {
        const int c = lane & 15, g = lane >> 4;
        const int key_k = tile * kDecodeTile + c / 4 * 8, key_v = tile * kDecodeTile + g * 8, mask = (1 << p.shift) - 1;
        int page_k = u.pages[min(key_k, u.length - 1) >> p.shift], page_v = u.pages[min(key_v, u.length - 1) >> p.shift];
        bad_k = (unsigned)page_k >= (unsigned)p.pages;
        bad_v = (unsigned)page_v >= (unsigned)p.pages;
        if (bad_k) page_k = 0;
        if (bad_v) page_v = 0;
        const char* at_k = u.K + page_k * p.k_page + ((key_k & mask) + c % 4) * p.k_row + g * 16;
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int s = 0; s < D / 32; ++s) k[mt][s] = *reinterpret_cast<const u4*>(at_k + mt * 4 * p.k_row + s * 64);
        const char* at_v = u.V + page_v * p.v_page + (key_v & mask) * p.v_row + c * (D / 8);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (D == 128) {
                const u4 w = *reinterpret_cast<const u4*>(at_v + i * p.v_row);
#pragma unroll
                for (int x = 0; x < 4; ++x) v[i][x] = w[x];
            } else {
                const u2 w = *reinterpret_cast<const u2*>(at_v + i * p.v_row);
#pragma unroll
                for (int x = 0; x < 2; ++x) v[i][x] = w[x];
            }
        }
    }
};

template <int D, bool BF16>
struct DecodeState {
    f4 o[D / 16];        // lane (c, g): head c, elements (4 g + i) * D / 16 + j of O in o[j][i]
    float m, l;          // running maximum of head c (in all lane groups alike), sum of the lane's own keys

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int j = 0; j < D / 16; ++j) o[j] = f4{0.f, 0.f, 0.f, 0.f};
        m = -INFINITY;
        l = 0.f;
    }

    __device__ __forceinline__ void add(const DecodeParams& p, const DecodeUnit& u, const u4 (&q)[D / 32], DecodeTile<D>& t, int tile, int lane) {
        const int g = lane >> 4, key0 = tile * kDecodeTile + g * 8;
        f4 s[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) s[mt] = decode_mfma<BF16>(t.k[mt][x], q[x], s[mt]);
#pragma unroll
        for (int mt = 0; mt < 2; ++mt) s[mt] *= p.c;
        const bool edge = tile * kDecodeTile < u.low || (tile + 1) * kDecodeTile > u.length;
        if (edge || __any(t.bad_v)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool seen = key0 + i >= u.low && key0 + i < u.length;
                s[i / 4][i % 4] = !seen ? -INFINITY : t.bad_v ? __builtin_nanf("") : s[i / 4][i % 4];
                if (!seen) {      // whatever the row holds, it takes no part: 0 * NaN would
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) t.v[i][x] = 0;
                }
            }
        }
        float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        if (__any(most > m)) {
            const float next = fmaxf(m, most), fade = next == -INFINITY ? 1.f : fast_exp2(m - next);
            m = next;
            l *= fade;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[j] *= fade;
        }
        // (nothing seen so far: any finite reference gives probabilities of 0)
        const float reference = (m == -INFINITY ? 0.f : m) - (BF16 ? 0.f : 12.f);
        u4 high, rest;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float a = fast_exp2(s[w / 2][w % 2 * 2] - reference), b = fast_exp2(s[w / 2][w % 2 * 2 + 1] - reference);
            l += a + b;
            high[w] = narrow<BF16>(a, b);
            rest[w] = narrow<BF16>(a - widen<BF16>(high[w], 0), b - widen<BF16>(high[w], 1));
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            u4 a;      // element j of the lane's pieces of the eight rows
#pragma unroll
            for (int w = 0; w < 4; ++w) a[w] = __builtin_amdgcn_perm(t.v[2 * w + 1][j / 2], t.v[2 * w][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
            o[j] = decode_mfma<BF16>(a, high, o[j]);
            o[j] = decode_mfma<BF16>(a, rest, o[j]);
        }
    }
};

__device__ __forceinline__ void store_o(char* to, int dtype, f4 x) {
    if (dtype == SAWATTN_F32) *reinterpret_cast<f4*>(to) = x;
    else if (dtype == SAWATTN_BF16) *reinterpret_cast<u2*>(to) = u2{narrow<true>(x[0], x[1]), narrow<true>(x[2], x[3])};
    else *reinterpret_cast<u2*>(to) = u2{narrow<false>(x[0], x[1]), narrow<false>(x[2], x[3])};
}

template <int D, bool BF16>
__global__ __launch_bounds__(kDecodeThreads) void decode_kernel(DecodeParams p) {
    constexpr int kPitch = D + 4;      // (rows of 16 lanes' pieces start in different banks)
    __shared__ __align__(16) float o_of[kDecodeWaves][kDecodeHeads][kPitch];
    __shared__ float m_of[kDecodeWaves][kDecodeHeads], l_of[kDecodeWaves][kDecodeHeads];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), c = lane & 15, g = lane >> 4;
    const int grid = gridDim.x;

    const DecodeShares shares(p, lane, grid, -1);
    long long at = blockIdx.x * shares.share;
    const long long end = min(at + shares.share, shares.total);
    if (at >= end) return;

    // the request that holds tile `at`, and how many tiles of the requests go before it
    int r = 0;
    long long before = 0;
    const long long wanted = divide(at, p.units);
    for (int r0 = 0; r0 < p.R; r0 += 64) {
        const int n = r0 + lane < p.R ? DecodeRequest(p, p.lengths[r0 + lane]).tiles : 0;
        long long upto = n;
#pragma unroll
        for (int step = 1; step < 64; step *= 2) {
            const long long x = __shfl_up(upto, step);
            if (lane >= step) upto += x;
        }
        const unsigned long long found = __ballot(before + upto > wanted);
        if (found) {
            const int here = __builtin_ctzll(found);
            r = r0 + here;
            before += __shfl(upto - n, here);
            break;
        }
        before += __shfl(upto, 63);
    }
    r = __builtin_amdgcn_readfirstlane(r);
    DecodeRequest request(p, p.lengths[r]);
    const long long inside = at - before * p.units;      // below units * tiles of the request
    int unit = (int)divide(inside, request.tiles);
    int t0 = (int)(inside - (long long)unit * request.tiles);
    unit = __builtin_amdgcn_readfirstlane(unit);
    t0 = __builtin_amdgcn_readfirstlane(t0);
    int left = __builtin_amdgcn_readfirstlane((int)(end - at));      // tiles of the workgroup still to do

    while (left > 0) {
        const int t1 = min(request.tiles, t0 + left);
        const int kv_head = unit / p.head_groups, head0 = (unit - kv_head * p.head_groups) * kDecodeHeads;
        const int heads = min(kDecodeHeads, p.group - head0);
        const char* q_row = p.Q + r * p.q_request + (long long)(kv_head * p.group + head0) * p.q_head;
        u4 q[D / 32];
#pragma unroll
        for (int x = 0; x < D / 32; ++x) q[x] = c < heads ? *reinterpret_cast<const u4*>(q_row + c * p.q_head + x * 64 + g * 16) : u4{0, 0, 0, 0};
        const DecodeUnit u = {p.K + kv_head * p.k_head, p.V + kv_head * p.v_head, p.table + r * p.table_stride, request.low, request.length};
        DecodeState<D, BF16> state;
        state.clear();
        for (int t = request.first + t0 + wave; t < request.first + t1; t += kDecodeWaves) {
            DecodeTile<D> tile;
            tile.load(p, u, t, lane);
            state.add(p, u, q, tile, t, lane);
        }
        state.l += __shfl_xor(state.l, 16);
        state.l += __shfl_xor(state.l, 32);
        if (c < heads) {
            if (g == 0) {
                m_of[wave][c] = state.m;
                l_of[wave][c] = state.l;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < D / 16; j += 4)
                    *reinterpret_cast<f4*>(&o_of[wave][c][(4 * g + i) * (D / 16) + j]) = f4{state.o[j][i], state.o[j + 1][i], state.o[j + 2][i], state.o[j + 3][i]};
        }
        __syncthreads();
        const bool whole = t0 == 0 && t1 == request.tiles;
        const int place = 2 * blockIdx.x + (t0 == 0 ? 1 : 0);      // of a part: a unit's first part ends its workgroup's work, others begin it
        for (int e = tid; e < heads * (D / 4); e += kDecodeThreads) {
            const int head = e / (D / 4), at4 = e % (D / 4) * 4;
            float m = m_of[0][head];
#pragma unroll
            for (int w = 1; w < kDecodeWaves; ++w) m = fmaxf(m, m_of[w][head]);
            const float reference = m == -INFINITY ? 0.f : m;
            float l = 0.f;
            f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < kDecodeWaves; ++w) {
                const float f = fast_exp2(m_of[w][head] - reference);
                l += f * l_of[w][head];
                o += f * *reinterpret_cast<const f4*>(&o_of[w][head][at4]);
            }
            if (whole) {
                const long long row = r * p.o_request + (long long)(kv_head * p.group + head0 + head) * p.o_head;
                store_o(p.O + row + at4 * (p.o_dtype == SAWATTN_F32 ? 4 : 2), p.o_dtype, o / l);
            } else {
                *reinterpret_cast<f4*>(p.parts + ((long long)place * p.heads_kept + head) * D + at4) = o;
                if (at4 == 0) p.part_sums[place * p.heads_kept + head] = f2{m, l};
            }
        }
        __syncthreads();
        left -= t1 - t0;
        t0 = 0;
        if (++unit == p.units && left > 0) {      // (with tiles left there is a request left that has some)
            unit = 0;
            do request = DecodeRequest(p, p.lengths[++r]);
            while (request.tiles == 0);
        }
    }
}

// One workgroup per row of O: adds up the parts of rows that several workgroups shared, and clears those of empty requests.  A group of
// D / 4 threads goes over every (1024 / D)-th part.
template <int D>
__global__ __launch_bounds__(kDecodeThreads) void decode_join_kernel(DecodeParams p, int grid, int H) {
    constexpr int kAcross = D / 4, kGroups = kDecodeThreads / kAcross;
    __shared__ f4 o_of[kGroups][kAcross];
    __shared__ float m_of[kGroups], l_of[kGroups];
    const int r = blockIdx.x / H, h = blockIdx.x - r * H, tid = threadIdx.x, a = tid % kAcross, of = tid / kAcross;
    const DecodeRequest request(p, p.lengths[r]);
    char* const to = p.O + r * p.o_request + h * p.o_head + a * (p.o_dtype == SAWATTN_F32 ? 16 : 8);
    if (request.tiles == 0) {
        if (of == 0) store_o(to, p.o_dtype, f4{0.f, 0.f, 0.f, 0.f});
        return;
    }
    const DecodeShares shares(p, tid & 63, grid, r);
    const int kv_head = h / p.group, inside = h - kv_head * p.group, unit = kv_head * p.head_groups + inside / kDecodeHeads, head = inside % kDecodeHeads;
    const long long begin = shares.before * p.units + (long long)unit * request.tiles;
    const int w0 = (int)divide(begin, shares.share), w1 = (int)divide(begin + request.tiles - 1, shares.share);
    if (w0 == w1) return;
    float m = -INFINITY, l = 0.f;
    f4 o = {0.f, 0.f, 0.f, 0.f};
    for (int w = w0 + of; w <= w1; w += kGroups) {
        const long long place = (long long)(2 * w + (w == w0 ? 1 : 0)) * p.heads_kept + head;
        const f2 sums = p.part_sums[place];
        const f4 part = *reinterpret_cast<const f4*>(p.parts + place * D + a * 4);
        const float next = fmaxf(m, sums[0]), reference = next == -INFINITY ? 0.f : next;
        const float fade = fast_exp2(m - reference), f = fast_exp2(sums[0] - reference);
        l = l * fade + sums[1] * f;
        o = o * fade + part * f;
        m = next;
    }
    o_of[of][a] = o;
    if (a == 0) {
        m_of[of] = m;
        l_of[of] = l;
    }
    __syncthreads();
    if (of != 0) return;
    m = m_of[0];
#pragma unroll
    for (int i = 1; i < kGroups; ++i) m = fmaxf(m, m_of[i]);
    const float reference = m == -INFINITY ? 0.f : m;
    l = 0.f;
    o = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        const float f = fast_exp2(m_of[i] - reference);
        l += f * l_of[i];
        o += f * o_of[i][a];
    }
    store_o(to, p.o_dtype, o / l);
}

// The launch for a problem, from what the host knows.
struct DecodePlan {
    int group, head_groups, units, heads_kept, grid;
};

int decode_plan(const sawattn_kv_cache* cache, int R, int H, int max_pages, DecodePlan* out) {
    if (R <= 0 || H <= 0 || max_pages <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "R, H and max_pages must be positive");
    if ((long long)R * H >= (1LL << 31)) return fail(SAWATTN_ERR_INVALID_ARG, "R*H must be below 2^31");
    if (H % cache->heads) return fail(SAWATTN_ERR_INVALID_ARG, "H must be a multiple of the cache's heads");
    const long long capacity = (long long)max_pages * cache->page_size;
    if (capacity >= (1LL << 31)) return fail(SAWATTN_ERR_INVALID_ARG, "max_pages*page_size must be below 2^31");
    out->group = H / cache->heads;
    out->head_groups = (out->group + kDecodeHeads - 1) / kDecodeHeads;
    out->units = out->head_groups * cache->heads;
    out->heads_kept = std::min(out->group, kDecodeHeads);
    const double most = (double)R * out->units * ((capacity + kDecodeTile - 1) / kDecodeTile);      // tiles, with every table full
    if (most >= 1e12) return fail(SAWATTN_ERR_INVALID_ARG, "R*H*max_pages*page_size is too large");
    out->grid = (int)std::max(1.0, std::min((double)kDecodeGrid, std::ceil(most / kDecodeLeast)));
    return SAWATTN_OK;
}

template <int D, bool BF16>
int launch_decode(const DecodeParams& p, int grid, int H, hipStream_t stream) {
    hipLaunchKernelGGL((decode_kernel<D, BF16>), dim3(grid), dim3(kDecodeThreads), 0, stream, p);
    const int rc = launched("attn_decode");
    if (rc != SAWATTN_OK) return rc;
    hipLaunchKernelGGL((decode_join_kernel<D>), dim3(p.R * H), dim3(kDecodeThreads), 0, stream, p, grid, H);
    return launched("attn_decode");
}

size_t decode_bytes(const DecodePlan& plan, int d) { return (size_t)2 * plan.grid * plan.heads_kept * (d + 2) * sizeof(float); }

}  // namespace sawattn

extern "C" {

int attn_decode_workspace_bytes(const sawattn_kv_cache* cache, int R, int H, int max_pages, size_t* bytes) {
    using namespace sawattn;
    if (!bytes) return fail(SAWATTN_ERR_INVALID_ARG, "bytes must be non-null");
    int rc = check_cache(cache, false);
    if (rc != SAWATTN_OK) return rc;
    DecodePlan plan;
    rc = decode_plan(cache, R, H, max_pages, &plan);
    if (rc != SAWATTN_OK) return rc;
    *bytes = decode_bytes(plan, cache->d);
    return SAWATTN_OK;
}

int attn_decode(const void* Q, int64_t q_request, int64_t q_head, void* O, int64_t o_request, int64_t o_head, int o_dtype,
                const sawattn_kv_cache* cache, const int32_t* table, int64_t table_stride, int max_pages,
                const int32_t* lengths, int R, int H, float scale, int window, void* workspace, size_t workspace_bytes,
                void* hip_stream) {
    using namespace sawattn;
    int rc = check_cache(cache, true);
    if (rc != SAWATTN_OK) return rc;
    DecodePlan plan;
    rc = decode_plan(cache, R, H, max_pages, &plan);
    if (rc != SAWATTN_OK) return rc;
    if (!Q || !O || !table || !lengths || !workspace)
        return fail(SAWATTN_ERR_INVALID_ARG, "Q, O, table, lengths and workspace must be non-null");
    if (((uintptr_t)Q | (uintptr_t)O | (uintptr_t)workspace) & 15u)
        return fail(SAWATTN_ERR_INVALID_ARG, "Q, O and workspace must be 16-byte aligned");
    if (((uintptr_t)table | (uintptr_t)lengths) & 3u) return fail(SAWATTN_ERR_INVALID_ARG, "table and lengths must be 4-byte aligned");
    if (o_dtype != SAWATTN_F16 && o_dtype != SAWATTN_BF16 && o_dtype != SAWATTN_F32)
        return fail(SAWATTN_ERR_INVALID_ARG, "o_dtype must be SAWATTN_F16, SAWATTN_BF16 or SAWATTN_F32");
    if (!std::isfinite(scale)) return fail(SAWATTN_ERR_INVALID_ARG, "scale must be finite");
    if (window < 0) return fail(SAWATTN_ERR_INVALID_ARG, "window must not be negative");
    if (table_stride < max_pages || (double)table_stride * R >= 1e18)
        return fail(SAWATTN_ERR_INVALID_ARG, "table_stride must be at least max_pages");
    const int d = cache->d;
    if (!good_stride(q_request, R) || !good_stride(q_head, H) || !good_stride(o_request, R) || !good_stride(o_head, H))
        return fail(SAWATTN_ERR_INVALID_ARG, "strides of Q and O must be multiples of 8, not negative");
    if ((R > 1 && o_request < d) || (H > 1 && o_head < d)) return fail(SAWATTN_ERR_INVALID_ARG, "strides of O must be at least d");
    if (workspace_bytes < decode_bytes(plan, d))
        return fail(SAWATTN_ERR_INVALID_ARG, "workspace is smaller than attn_decode_workspace_bytes reports");
    const int o_size = o_dtype == SAWATTN_F32 ? 4 : 2;
    auto extent = [](int n, int64_t stride) { return n > 1 ? (unsigned long long)(n - 1) * stride : 0ull; };
    const Range o(O, o_size * (extent(R, o_request) + extent(H, o_head) + d));
    const Range scratch(workspace, decode_bytes(plan, d));
    const Range in[] = {
        {Q, 2 * (extent(R, q_request) + extent(H, q_head) + d)},
        {cache->k, 2 * (extent(cache->pages, cache->k_page) + extent(cache->heads, cache->k_head) + extent(cache->page_size, cache->k_row) + d)},
        {cache->v, 2 * (extent(cache->pages, cache->v_page) + extent(cache->heads, cache->v_head) + extent(cache->page_size, cache->v_row) + d)},
        {table, 4 * (extent(R, table_stride) + max_pages)}, {lengths, 4ull * R}};
    for (const Range& i : in)
        if (o.meets(i) || scratch.meets(i)) return fail(SAWATTN_ERR_INVALID_ARG, "O and workspace must not overlap what is read");
    if (o.meets(scratch)) return fail(SAWATTN_ERR_INVALID_ARG, "O must not overlap the workspace");

    DecodeParams p{};
    p.Q = static_cast<const char*>(Q); p.q_request = 2 * q_request; p.q_head = 2 * q_head;
    p.O = static_cast<char*>(O); p.o_request = o_size * o_request; p.o_head = o_size * o_head; p.o_dtype = o_dtype;
    p.K = static_cast<const char*>(cache->k); p.V = static_cast<const char*>(cache->v);
    p.k_page = 2 * cache->k_page; p.k_head = 2 * cache->k_head; p.k_row = 2 * cache->k_row;
    p.v_page = 2 * cache->v_page; p.v_head = 2 * cache->v_head; p.v_row = 2 * cache->v_row;
    p.table = table; p.table_stride = table_stride; p.lengths = lengths;
    p.parts = static_cast<float*>(workspace);
    p.part_sums = reinterpret_cast<f2*>(p.parts + (size_t)2 * plan.grid * plan.heads_kept * d);
    p.c = (float)((double)scale * 1.4426950408889634074);
    p.R = R; p.capacity = max_pages * cache->page_size; p.window = window; p.pages = cache->pages; p.shift = page_shift(cache->page_size);
    p.group = plan.group; p.head_groups = plan.head_groups; p.units = plan.units; p.heads_kept = plan.heads_kept;
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const bool bf = cache->dtype == SAWATTN_BF16;
    if (d == 128) return bf ? launch_decode<128, true>(p, plan.grid, H, stream) : launch_decode<128, false>(p, plan.grid, H, stream);
    return bf ? launch_decode<64, true>(p, plan.grid, H, stream) : launch_decode<64, false>(p, plan.grid, H, stream);
}

}  // extern "C"
