// attn_decode: attention of one new token per request over a paged key-value cache.
//
//   s_j = scale q . k_j,  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m)   over the visible rows j of a request
//
// Bound by memory: every key and value is read once, for 4 d flops per query head that shares it.  A unit is a request and a key/value
// head, with up to 16 of its query heads; for more there is a set of workgroups for every 16 (a head group).
//
// Who does what.  Where a unit is short (decode_plan) a workgroup of one to eight wavefronts takes all of it: one launch.  Else the units' rows are cut into
// steps of 128, and the steps of all units, one behind the other, are dealt out evenly: workgroup w takes `share` of them from w * share on, whatever the
// lengths are, so that one long request and many short ones load the chip alike and the host needs to know no length.  A workgroup ends at
// most two units unfinished, its first and its last; of those it leaves (m, sum, O) of its part in one of its two places in the workspace,
// and a second kernel joins them.  Measured (here and below: calls captured into a graph, inputs changing; 16 x 32768, ungrouped): 256, 512, 1024 and 2048 workgroups 660, 660, 670 and 690 us; ragged requests want
// two workgroups to a compute unit, so that one loads while the other ends a unit (64 requests up to 8192: 95 us, one of eight wavefronts 103).
//
// Within a workgroup every wavefront takes tiles of 32 keys of its own, with its own running maximum and sum; they are added up in LDS at the
// unit's end.  Products run on 16x16x32 MFMAs, transposed: S^T = K Q^T, O^T = V^T P^T with the 16 columns the query heads (columns without
// one are computed and dropped: the matrix cores idle anyway).  K passes through LDS, by direct loads of whole rows: read from memory in
// the operands' order, 64 bytes of 16 rows at a time, it took 5 % longer.  In the result a lane (c = lane % 16, g = lane / 16) holds eight scores of
// head c: rows 4 g + i of two MFMAs.  Row 4 g + i stands for key 4 i + g of 16, so that the lane's eight keys are those of which it
// has to hold the probabilities as B operand of the second product: they stay where they are.  V comes as rows 4 i + g, 16 bytes (8 at d = 64)
// of each per lane, four whole rows per load, and never leaves the registers: pairs of rows are interleaved (v_perm) into A operands, whose MFMA j
// has elements j, j + D/16, ... of V.
//
// The probabilities enter the second product as sums of three 16-bit numbers (DecodePieces), for which the matrix cores have time.  Binary16 ones are
// scaled by 2^15 for the sake of small ones.
//
// K and V are read with non-temporal loads (7.1 instead of 6.3 TB/s for a kernel that only reads).  Measured with the products taken out,
// the loads of 16 x 32768 take 655 us (pages of 16 rows in any order; of 256 rows: 645), with them 660: 6.5 TB/s.  Loading a tile ahead, in
// registers, gave nothing: four wavefronts on each of four SIMDs keep enough on its way.
namespace sawattn {

constexpr int kDecodeWaves = 4;                                  // of a workgroup that shares units with others
constexpr int kDecodeTile = 32;                                  // keys a wavefront takes at a time
constexpr int kDecodeStep = kDecodeTile * kDecodeWaves;          // keys such a workgroup takes at a time: what is dealt out
constexpr int kDecodeHeads = 16;                                 // query heads of a unit
constexpr long long kDecodeDirectFew = 1 << 18, kDecodeDirectMany = 1 << 20;      // bytes of K and V of a unit at most, with fewer or more units than compute units
constexpr int kDecodeGrid = 1024;                                // workgroups that share units (half as many at d = 128), in all sets; eight a set at least
constexpr int kDecodeUnits = 256;                                // compute units: up to as many workgroups of one step, then of two at least

struct DecodeParams {
    const char* Q;
    char* O;
    long long q_request, q_head, o_request, o_head;      // bytes
    const char* K;
    const char* V;
    long long k_page, k_head, v_page, v_head;            // bytes
    unsigned k_row, v_row;
    const int* table;
    long long table_stride;
    const int* lengths;
    float* parts;        // workspace: [2 * grid][heads_kept][D] of O
    f2* part_sums;       // [2 * grid][heads_kept] of (maximum, sum)
    int4* begun;         // [grid] the unit that the workgroup leaves for others to end: (request, unit, workgroup that ends it, 0); request -1: none
    float c;             // scale * log2(e)
    int o_dtype, R, capacity, window, pages, shift;
    int group;           // query heads per key/value head
    int head_groups;     // by which a key/value head's query heads go, 16 at a time
    int units;           // per request: key/value heads
    int workgroups;      // for each head group
    int heads_kept;      // of a unit: min(group, 16)
};

// Workgroups come in one set for each head group, which share their keys and values: the same workgroup of all sets on one XCD (blocks go
// round the eight of them), one behind the other, so that what the first brings into the L2 the others find there (16 requests x 30000 keys, one
// key head: 16 query heads 52 us, 64 102; read anew by every set 161).
__device__ __forceinline__ int block_of(const DecodeParams& p, int workgroup, int head_group) {
    return p.head_groups == 1 ? workgroup : (workgroup / 8 * p.head_groups + head_group) * 8 + workgroup % 8;
}

struct DecodeRequest {
    int length, low, first, steps;      // visible rows low .. length - 1, in steps from `first` on
    __device__ __forceinline__ DecodeRequest(const DecodeParams& p, int given) {
        length = min(max(given, 0), p.capacity);
        low = p.window ? max(length - p.window, 0) : 0;
        first = low / kDecodeStep;
        steps = length ? (length - 1) / kDecodeStep - first + 1 : 0;
    }
};

// How the steps are dealt out, from the lengths alone: what workgroup `wg` of `grid` has to do.  Every wavefront works it out for itself.
struct DecodeShare {
    int share;                 // steps of a workgroup
    int left;                  // of this one: none if not positive
    int r, unit, t0;           // the first one: request, unit of the request, step of the unit
    int length;                // lengths[r]
    __device__ __forceinline__ DecodeShare(const DecodeParams& p, int lane, int wg, int grid) {
        // the first 64 lengths stay in registers: mostly there are no more, and a second trip to memory would cost as much as a step
        const int given0 = lane < p.R ? p.lengths[lane] : 0;
        int all = DecodeRequest(p, given0).steps;
        for (int i = lane + 64; i < p.R; i += 64) all += DecodeRequest(p, p.lengths[i]).steps;
        const int total = __builtin_amdgcn_readlane(lanes_upto(all), 63) * p.units;
        share = max((int)(((unsigned)total + grid - 1) / (unsigned)grid), total > kDecodeUnits / p.head_groups ? 2 : 1);
        const int at = min(wg, grid - 1) * share;      // (below the total and twice the grid)
        left = wg < grid ? min(share, total - at) : 0;
        r = unit = t0 = length = 0;
        if (left <= 0) return;
        const int wanted = (unsigned)at / (unsigned)p.units;
        int before = 0;      // steps of the requests in front
        for (int r0 = 0; r0 < p.R; r0 += 64) {
            const int given = r0 == 0 ? given0 : r0 + lane < p.R ? p.lengths[r0 + lane] : 0;
            const int steps = DecodeRequest(p, given).steps, upto = lanes_upto(steps);
            const unsigned long long found = __ballot(before + upto > wanted);
            if (found) {
                const int here = __builtin_ctzll(found), of_request = __builtin_amdgcn_readlane(steps, here);
                r = r0 + here;
                length = __builtin_amdgcn_readlane(given, here);
                const int inside = at - (before + __builtin_amdgcn_readlane(upto, here) - of_request) * p.units;      // below units * steps of the request
                unit = (unsigned)inside / (unsigned)of_request;
                t0 = inside - unit * of_request;
                return;
            }
            before += __builtin_amdgcn_readlane(upto, 63);
        }
        left = 0;      // (not reached unless the lengths change meanwhile)
    }
};

template <bool BF16>
__device__ __forceinline__ f4 decode_mfma(u4 a, u4 b, f4 c) {
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}

// Two probabilities as sums of three 16-bit numbers each: cut off, not rounded, and what each leaves goes to the next, which holds all of their 24 bits
// (binary16: down to 2^-16 of the largest, below that to 2^-38 of it).  None of the three is zero or negative unless the probability is that
// small: the product of such a one with an infinite value would be no number, or the other infinity.
template <bool BF16>
struct DecodePieces {
    static constexpr int kCount = 3;
    unsigned word[kCount];
    __device__ __forceinline__ DecodePieces(float a, float b) {
        if constexpr (BF16) {      // eight bits at a time, of the next smaller number, so that something is left
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                const unsigned one = i + 1 < kCount ? 1u : 0u;
                const unsigned x = __builtin_elementwise_sub_sat(__builtin_bit_cast(unsigned, a), one), y = __builtin_elementwise_sub_sat(__builtin_bit_cast(unsigned, b), one);
                word[i] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                a -= __builtin_bit_cast(float, x & 0xffff0000u);
                b -= __builtin_bit_cast(float, y & 0xffff0000u);
            }
        } else {      // eleven bits; what is left is at least the smallest number there is, where the probability is
            const float least_a = fminf(a, 0x1p-24f), least_b = fminf(b, 0x1p-24f);
#pragma unroll
            for (int i = 0; i < kCount; ++i) {
                word[i] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(a, b));
                a = fmaxf(a - widen<false>(word[i], 0), least_a);
                b = fmaxf(b - widen<false>(word[i], 1), least_b);
            }
        }
    }
};

// The larger, and the sum, of x in the four lanes that hold a head.
__device__ __forceinline__ void lane_quarters(float x, float& one, float& other) {      // neighbouring rows of 16 lanes exchanged
    unsigned a = __builtin_bit_cast(unsigned, x), b = a;
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
    one = __builtin_bit_cast(float, a);
    other = __builtin_bit_cast(float, b);
}
__device__ __forceinline__ float head_max(float x) {
    float one, other;
    lane_quarters(x, one, other);
    return pair_max(fmaxf(one, other));
}
__device__ __forceinline__ float head_sum(float x) {
    float one, other;
    lane_quarters(x, one, other);
    return pair_sum(one + other);
}

// A tile's way through LDS and registers; lane constants.  16-byte pieces of a row of K change places in LDS (by exclusive or with the
// row's number: `turn`), so that the same piece of 16 rows lies in all banks; the lane that loads a piece fetches the one that belongs there.
// The 16 lanes that are served at a time are not those of one piece, and two of them meet in a bank: four cycles more for each read
// (1.05 million conflicts to 262144 reads of 1 x 131072 keys), in the shade of the loads from memory.
template <int D>
struct DecodeLane {
    static constexpr int kRowBytes = 2 * D, kLoads = kDecodeTile * kRowBytes / 1024, kPieces = kRowBytes / 16, kRowsPerLoad = 64 / kPieces;
    int c, g;
    unsigned k_row, k_piece;      // the lane's row and piece of a load of K, in bytes
    unsigned v_from;              // byte offset of its piece in the four rows of a load of V
    int k_at;                     // in the tile in LDS: its A operands of the first 16 keys, first 32 elements
    __device__ __forceinline__ DecodeLane(const DecodeParams& p, int lane) {
        c = lane & 15;
        g = lane >> 4;
        k_row = lane / kPieces * p.k_row;
        k_piece = (lane % kPieces ^ turn(lane / kPieces)) * 16;
        v_from = g * p.v_row + c * (D / 8);
        const int mine = 4 * (c & 3) + (c >> 2);      // of 16 keys the one whose scores are row c of the product
        k_at = mine * kRowBytes + (g ^ turn(mine)) * 16;
    }
    static __device__ __forceinline__ int turn(int row) { return D == 128 ? row & 15 : row >> 1 & 7; }
    // Load i of a tile fetches rows from i * kRowsPerLoad on, whose numbers have no bit in common with a lane's row in them.
    __device__ __forceinline__ unsigned k_from(int i) const { return k_row + (k_piece ^ turn(i * kRowsPerLoad) * 16); }
    // Elements 32 x .. of the operand are the lane's 16-byte pieces 4 x + g.
    __device__ __forceinline__ int k_operand(int x) const { return k_at ^ x * 64; }
};

// What a unit's tiles need of its request and head.
struct DecodeUnit {
    const char* K;
    const char* V;
    const __attribute__((address_space(4))) int* pages;      // (through the scalar cache: a tile's two pages are the wavefront's)
    int low, length;
};

struct DecodePages {      // of the two halves of a tile
    int half[2];
    __device__ __forceinline__ DecodePages(const DecodeParams& p, const DecodeUnit& u, int tile) {
#pragma unroll
        for (int i = 0; i < 2; ++i) half[i] = u.pages[min(tile * kDecodeTile + i * 16, u.length - 1) >> p.shift];
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

    // BRIEF: of a tile at an edge only the rows are read that are visible, in loads of four or eight (where requests are short, edges are most of
    // what there is; else the branches cost more than the rows: 64 ragged requests up to 8192, 94 and 97 us).
    template <bool BRIEF>
    __device__ __forceinline__ void add(const DecodeParams& p, const DecodeLane<D>& lane, const DecodeUnit& u, const u4 (&q)[D / 32], const DecodePages& pages, int tile,
                                        LDS_PTR(char) lds) {
        using L = DecodeLane<D>;
        const int mask = (1 << p.shift) - 1, key0 = tile * kDecodeTile;
        const bool edge = key0 < u.low || key0 + kDecodeTile > u.length;
        bool bad[2];
        unsigned v[8][D / 32];
#pragma unroll
        for (int half = 0; half < 2; ++half) bad[half] = (unsigned)pages.half[half] >= (unsigned)p.pages;
        auto load = [&](auto all) {
            constexpr bool ALL = decltype(all)::value;
            auto wanted = [&](int first, int rows) { return ALL || (key0 + first < u.length && key0 + first + rows > u.low); };
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int page = bad[half] ? 0 : pages.half[half], row = (key0 + half * 16) & mask;
                const char* k = u.K + page * p.k_page + (long long)row * p.k_row;
#pragma unroll
                for (int i = 0; i < L::kLoads / 2; ++i)
                    if (wanted(half * 16 + i * L::kRowsPerLoad, L::kRowsPerLoad))
                        load_to_lds_16B_nt(k + (long long)i * L::kRowsPerLoad * p.k_row, lane.k_from(i),
                                           (unsigned)(uintptr_t)lds + (half * (L::kLoads / 2) + i) * 1024);
            }
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const int page = bad[half] ? 0 : pages.half[half], row = (key0 + half * 16) & mask;
                const char* from = u.V + page * p.v_page + (long long)row * p.v_row;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const char* at = from + (long long)i * 4 * p.v_row + lane.v_from;
                    typedef unsigned words __attribute__((ext_vector_type(D / 32)));
                    words w = {};
                    if (wanted(half * 16 + i * 4, 4)) w = __builtin_nontemporal_load(reinterpret_cast<const words*>(at));
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) v[half * 4 + i][x] = w[x];
                }
            }
        };
        if (BRIEF && edge) {
            load(std::false_type{});
            wait_tile_landed();
        } else {
            load(std::true_type{});
            // K has landed when no more are on their way than the eight loads of V behind it (1 x 200 keys 4.08 -> 3.93 us, 64 ragged 94 -> 92.7)
            asm volatile("s_waitcnt vmcnt(8)" ::: "memory");
        }
        f4 s[2] = {f4{0.f, 0.f, 0.f, 0.f}, f4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int half = 0; half < 2; ++half)
                s[half] = decode_mfma<BF16>(*(LDS_PTR(const u4))(lds + lane.k_operand(x) + half * 16 * L::kRowBytes), q[x], s[half]);
#pragma unroll
        for (int half = 0; half < 2; ++half) s[half] *= p.c;
        if (edge || bad[0] || bad[1]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = key0 + 4 * i + lane.g;
                const bool seen = key >= u.low && key < u.length;
                s[i / 4][i % 4] = !seen ? -INFINITY : bad[i / 4] ? __builtin_nanf("") : s[i / 4][i % 4];
                if (!seen) {      // whatever the row holds, it takes no part: 0 * NaN would
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) v[i][x] = 0;
                }
            }
        }
        float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        most = head_max(most);
        if (__any(most > m)) {
            const float next = fmaxf(m, most), fade = next == -INFINITY ? 1.f : fast_exp2(m - next);
            m = next;
            l *= fade;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[j] *= fade;
        }
        // (nothing seen so far: any finite reference gives probabilities of 0)
        const float reference = (m == -INFINITY ? 0.f : m) - (BF16 ? 0.f : 15.f);
        using Pieces = DecodePieces<BF16>;
        u4 piece[Pieces::kCount];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float a = fast_exp2(s[w / 2][w % 2 * 2] - reference), b = fast_exp2(s[w / 2][w % 2 * 2 + 1] - reference);
            l += a + b;
            const Pieces pieces(a, b);
#pragma unroll
            for (int i = 0; i < Pieces::kCount; ++i) piece[i][w] = pieces.word[i];
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            u4 a;      // element j of the lane's pieces of its eight rows
#pragma unroll
            for (int w = 0; w < 4; ++w) a[w] = __builtin_amdgcn_perm(v[2 * w + 1][j / 2], v[2 * w][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int i = 0; i < Pieces::kCount; ++i) o[j] = decode_mfma<BF16>(a, piece[i], o[j]);
        }
    }
};

__device__ __forceinline__ void store_o(char* to, int dtype, f4 x) {
    if (dtype == SAWATTN_F32) *reinterpret_cast<f4*>(to) = x;
    else if (dtype == SAWATTN_BF16) *reinterpret_cast<u2*>(to) = u2{narrow<true>(x[0], x[1]), narrow<true>(x[2], x[3])};
    else *reinterpret_cast<u2*>(to) = u2{narrow<false>(x[0], x[1]), narrow<false>(x[2], x[3])};
}

// DIRECT: a workgroup takes a unit, all of it; else what its number says of all units.
template <int D, bool BF16, int WAVES, bool DIRECT>
__global__ __launch_bounds__(64 * WAVES, 4) void decode_kernel(DecodeParams p) {
    static_assert(DIRECT || WAVES == kDecodeWaves, "shares are counted in steps of that many wavefronts");
    constexpr int kPitch = D + 4;      // floats of a head's O in LDS (rows of 16 lanes' pieces start in different banks)
    constexpr int kArea = kDecodeHeads * kPitch * 4;      // of a wavefront: its tile of K, and at a unit's end its O
    static_assert(kArea >= kDecodeTile * 2 * D, "a tile of K fits");
    __shared__ __align__(16) char area[WAVES][kArea];
    __shared__ float m_of[WAVES][kDecodeHeads], l_of[WAVES][kDecodeHeads];
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const DecodeLane<D> lane(p, tid & 63);

    int workgroup = blockIdx.x, head_group = 0;
    if (p.head_groups > 1) {
        const int eight = blockIdx.x / 8;
        head_group = eight % p.head_groups;
        workgroup = eight / p.head_groups * 8 + blockIdx.x % 8;      // (up to seven behind the last)
    }
    int r, unit, t0, left, share, length;
    if constexpr (DIRECT) {
        if (workgroup >= p.workgroups) return;
        r = workgroup / p.units;
        unit = workgroup - r * p.units;
        t0 = left = share = 0;
        length = __builtin_amdgcn_readfirstlane(p.lengths[r]);
    } else {
        const DecodeShare mine(p, tid & 63, workgroup, p.workgroups);
        r = mine.r; unit = mine.unit; t0 = mine.t0; left = mine.left; share = mine.share; length = mine.length;
        if (left <= 0) {
            if (tid == 0) p.begun[blockIdx.x] = int4{-1, 0, 0, 0};
            return;
        }
    }
    DecodeRequest request(p, length);

    do {
        const int t1 = min(request.steps, t0 + left);      // (not DIRECT)
        const int head0 = head_group * kDecodeHeads, heads = min(kDecodeHeads, p.group - head0);
        const char* q_row = p.Q + r * p.q_request + (long long)(unit * p.group + head0) * p.q_head;
        u4 q[D / 32];
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
            q[x] = lane.c < heads ? *reinterpret_cast<const u4*>(q_row + lane.c * p.q_head + x * 64 + lane.g * 16) : u4{0, 0, 0, 0};
        const DecodeUnit u = {p.K + unit * p.k_head, p.V + unit * p.v_head,
                              (const __attribute__((address_space(4))) int*)(uintptr_t)(p.table + r * p.table_stride), request.low, request.length};
        DecodeState<D, BF16> state;
        state.clear();
        // the wavefront's tiles, those that hold a visible row
        const int all_tiles = (request.length + kDecodeTile - 1) / kDecodeTile;
        int tile = DIRECT ? request.low / kDecodeTile + wave : (request.first + t0) * kDecodeWaves + wave;
        const int tiles = DIRECT ? all_tiles : min((request.first + t1) * kDecodeWaves, all_tiles);
        if (!DIRECT && (tile + 1) * kDecodeTile <= request.low) tile += kDecodeWaves;
        if (tile < tiles) {
            DecodePages pages(p, u, tile);
            do {
                const int next = tile + WAVES;
                const DecodePages ahead(p, u, next);      // (behind the last one the last page again)
                state.template add<DIRECT && WAVES < 8>(p, lane, u, q, pages, tile, (LDS_PTR(char))area[wave]);
                pages = ahead;
                tile = next;
            } while (tile < tiles);
        }
        state.l = head_sum(state.l);
        // (the lane's number made anew: what follows from it here is not to be kept in registers over the tiles)
        const int now = lane_now(), c = now & 15, g = now >> 4;
        if (c < heads) {
            if (g == 0) {
                m_of[wave][c] = state.m;
                l_of[wave][c] = state.l;
            }
            float* o = reinterpret_cast<float*>(area[wave]) + c * kPitch;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < D / 16; j += 4)
                    *reinterpret_cast<f4*>(o + (4 * g + i) * (D / 16) + j) = f4{state.o[j][i], state.o[j + 1][i], state.o[j + 2][i], state.o[j + 3][i]};
        }
        __syncthreads();
        const bool whole = DIRECT || (t0 == 0 && t1 == request.steps);
        const int place = 2 * blockIdx.x + (t0 == 0 ? 1 : 0);      // of a part: a unit's first part ends its workgroup's work, others begin it
        for (int e = wave * 64 + now; e < heads * (D / 4); e += 64 * WAVES) {
            const int head = e / (D / 4), at4 = e % (D / 4) * 4;
            float m = m_of[0][head];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) m = fmaxf(m, m_of[w][head]);
            const float reference = m == -INFINITY ? 0.f : m;
            float l = 0.f;
            f4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = fast_exp2(m_of[w][head] - reference);
                l += f * l_of[w][head];
                o += f * *reinterpret_cast<const f4*>(reinterpret_cast<const float*>(area[w]) + head * kPitch + at4);
            }
            if (whole) {
                const long long row = r * p.o_request + (long long)(unit * p.group + head0 + head) * p.o_head;
                store_o(p.O + row + at4 * (p.o_dtype == SAWATTN_F32 ? 4 : 2), p.o_dtype, request.length ? o / l : o);
            } else {
                *reinterpret_cast<f4*>(p.parts + ((long long)place * p.heads_kept + head) * D + at4) = o;
                if (at4 == 0) p.part_sums[place * p.heads_kept + head] = f2{m, l};
            }
        }
        left -= t1 - t0;
        if constexpr (DIRECT) return;
        if (left <= 0) {
            // what is missing of a unit begun here takes the workgroups behind this one, in whole shares
            if (tid == 0)
                p.begun[blockIdx.x] = int4{t0 == 0 && !whole ? r : -1, unit, min(workgroup + (request.steps - t1 + share - 1) / max(share, 1), p.workgroups - 1), 0};
            return;
        }
        __syncthreads();
        t0 = 0;
        if (++unit == p.units) {      // (with steps left there is a request left that has some, unless the lengths have changed meanwhile)
            unit = 0;
            do {
                if (++r == p.R) {
                    if (tid == 0) p.begun[blockIdx.x] = int4{-1, 0, 0, 0};
                    return;
                }
                request = DecodeRequest(p, __builtin_amdgcn_readfirstlane(p.lengths[r]));
            } while (request.steps == 0);
        }
    } while (true);
}

// Adds up the parts of the units that several workgroups shared, a workgroup for every two heads of each, and clears the rows of empty
// requests.  The threads that hold a head's elements, four each, go over every kGroups-th part, four parts on their way at a time.  It takes 4 us (6.5 where
// a unit has 64 parts), of which the parts are the least: launch, record of the unit, parts, result, one after the other.  (Two heads and 256 threads: 1 x 1000 keys 10.9 us in all, with
// four and 1024 11.2; parts fetched before the record is there: 0.3 to 1 us more.)
constexpr int kJoinThreads = 256, kJoinHeads = 2, kJoinAhead = 4;

template <int D>
__global__ __launch_bounds__(kJoinThreads) void decode_join_kernel(DecodeParams p, int H) {
    constexpr int kAcross = D / 4, kGroups = kJoinThreads / (kAcross * kJoinHeads);
    __shared__ f4 o_of[kGroups][kJoinHeads][kAcross];
    __shared__ f2 sums_of[kGroups][kJoinHeads];
    const int tid = threadIdx.x, a = tid % kAcross, of_head = tid / kAcross % kJoinHeads, group = tid / (kAcross * kJoinHeads);
    const int o_size = p.o_dtype == SAWATTN_F32 ? 4 : 2;
    const int4 unit = p.begun[blockIdx.x];
    if (blockIdx.y == 0)
        for (int r = blockIdx.x; r < p.R; r += gridDim.x)
            if (p.lengths[r] <= 0)
                for (int e = tid; e < H * kAcross; e += kJoinThreads)
                    store_o(p.O + r * p.o_request + e / kAcross * p.o_head + e % kAcross * 4 * o_size, p.o_dtype, f4{0.f, 0.f, 0.f, 0.f});
    if (unit.x < 0) return;
    int first = blockIdx.x, head_group = 0;
    if (p.head_groups > 1) {
        head_group = blockIdx.x / 8 % p.head_groups;
        first = blockIdx.x / 8 / p.head_groups * 8 + blockIdx.x % 8;
    }
    const int last = unit.z, head0 = head_group * kDecodeHeads, head = blockIdx.y * kJoinHeads + of_head;
    const bool mine = head < min(kDecodeHeads, p.group - head0);
    float m = -INFINITY, l = 0.f;
    f4 o = {0.f, 0.f, 0.f, 0.f};
    if (mine) {
        for (int w = first + group; w <= last; w += kGroups * kJoinAhead) {
            f2 sums[kJoinAhead];
            f4 part[kJoinAhead];
            float next = m;
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i) {
                const int at = min(w + i * kGroups, last);
                const long long place = (long long)(2 * block_of(p, at, head_group) + (at == first ? 1 : 0)) * p.heads_kept + head;
                sums[i] = p.part_sums[place];
                part[i] = *reinterpret_cast<const f4*>(p.parts + place * D + a * 4);
            }
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i) next = fmaxf(next, sums[i][0]);
            const float reference = next == -INFINITY ? 0.f : next, fade = fast_exp2(m - reference);
            l *= fade;
            o *= fade;
#pragma unroll
            for (int i = 0; i < kJoinAhead; ++i)
                if (w + i * kGroups <= last) {
                    const float f = fast_exp2(sums[i][0] - reference);
                    l += sums[i][1] * f;
                    o += part[i] * f;
                }
            m = next;
        }
        o_of[group][of_head][a] = o;
        if (a == 0) sums_of[group][of_head] = f2{m, l};
    }
    __syncthreads();
    if (group != 0 || !mine) return;
#pragma unroll
    for (int i = 1; i < kGroups; ++i) m = fmaxf(m, sums_of[i][of_head][0]);
    const float reference = m == -INFINITY ? 0.f : m;
    l = 0.f;
    o = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
        const float f = fast_exp2(sums_of[i][of_head][0] - reference);
        l += f * sums_of[i][of_head][1];
        o += f * o_of[i][of_head][a];
    }
    store_o(p.O + unit.x * p.o_request + (long long)(unit.y * p.group + head0 + head) * p.o_head + a * 4 * o_size, p.o_dtype, o / l);
}

// The launch for a problem, from what the host knows.
struct DecodePlan {
    int group, head_groups, units, heads_kept, workgroups, grid;
    int seen;         // rows of a unit, with every table full
    bool direct;
};

int decode_plan(const sawattn_kv_cache* cache, int R, int H, int max_pages, int window, DecodePlan* out) {
    if (R <= 0 || H <= 0 || max_pages <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "R, H and max_pages must be positive");
    if ((long long)R * H >= (1LL << 22)) return fail(SAWATTN_ERR_INVALID_ARG, "R*H must be below 2^22");      // (a launch has fewer than 2^32 threads)
    if (H % cache->heads) return fail(SAWATTN_ERR_INVALID_ARG, "H must be a multiple of the cache's heads");
    const long long capacity = (long long)max_pages * cache->page_size;
    if (capacity > (1LL << 30)) return fail(SAWATTN_ERR_INVALID_ARG, "max_pages*page_size must be at most 2^30");
    out->group = H / cache->heads;
    out->head_groups = (out->group + kDecodeHeads - 1) / kDecodeHeads;
    out->units = cache->heads;
    out->heads_kept = std::min(out->group, kDecodeHeads);
    out->seen = (int)(window > 0 ? std::min<long long>(capacity, window) : capacity);
    const double most = (double)R * out->units * ((capacity + kDecodeStep - 1) / kDecodeStep);      // steps
    if (most >= 2147483648.0 - 2.0 * kDecodeGrid)
        return fail(SAWATTN_ERR_INVALID_ARG, "R*heads*ceil(max_pages*page_size/128) must be below 2^31 - 2048");
    // One workgroup reads about 55 GB/s, the second kernel costs 6 us and more with the 2 us in front of it.  Few units: up to 500 keys at d = 128 take 8.5 us in one launch,
    // in two 9; 1000 keys 12.5 and 9.4.  Units for every compute unit and more: 256 requests of 1000 keys, 8 heads: 170 and 190 us, 128 ragged
    // requests up to 2000: 57 and 62.
    const long long units = (long long)R * out->units, bytes = 4LL * out->seen * cache->d, sets = out->head_groups;
    out->direct = bytes <= (units * sets >= kDecodeUnits ? kDecodeDirectMany : kDecodeDirectFew);
    const long long resident = (cache->d == 128 ? kDecodeGrid / 2 : kDecodeGrid) / sets, workgroups = out->direct ? units : std::min<long long>((long long)most, std::max(8LL, resident));
    const long long grid = sets == 1 ? workgroups : (workgroups + 7) / 8 * 8 * sets;      // (below 2^22 + 7 * 2^18)
    out->workgroups = (int)workgroups;
    out->grid = (int)grid;
    return SAWATTN_OK;
}

template <int D, bool BF16>
int launch_decode(const DecodeParams& p, const DecodePlan& plan, int H, hipStream_t stream) {
    if (plan.direct) {
        // A wavefront to a tile, up to eight of them; half as many where there are four units and more for every compute unit.  Measured with one
        // wavefront, with two and with eight, two tiles at most: 149 requests of 4 rows, 16 key/value heads 7.8, 9.5, 21.2 us; one of 60 rows, 8 heads
        // 6.0, 4.5, 4.7; 256 of 60 rows 14.2, 14.1, 20.5.  With two, four and eight, four tiles: 8 of 120 rows 6.3, 5.3, 5.5; 256 of 120 rows 24.2, 23.9, 29.7.
        const int tiles = (plan.seen + kDecodeTile - 1) / kDecodeTile, wanted = plan.grid >= 4 * kDecodeUnits ? (tiles + 1) / 2 : tiles;
        if (wanted <= 1) hipLaunchKernelGGL((decode_kernel<D, BF16, 1, true>), dim3(plan.grid), dim3(64), 0, stream, p);
        else if (wanted <= 2) hipLaunchKernelGGL((decode_kernel<D, BF16, 2, true>), dim3(plan.grid), dim3(128), 0, stream, p);
        else if (wanted <= 4) hipLaunchKernelGGL((decode_kernel<D, BF16, 4, true>), dim3(plan.grid), dim3(256), 0, stream, p);
        else hipLaunchKernelGGL((decode_kernel<D, BF16, 8, true>), dim3(plan.grid), dim3(512), 0, stream, p);
        return launched("attn_decode");
    }
    hipLaunchKernelGGL((decode_kernel<D, BF16, kDecodeWaves, false>), dim3(plan.grid), dim3(64 * kDecodeWaves), 0, stream, p);
    const int rc = launched("attn_decode");
    if (rc != SAWATTN_OK) return rc;
    hipLaunchKernelGGL((decode_join_kernel<D>), dim3(plan.grid, (plan.heads_kept + kJoinHeads - 1) / kJoinHeads), dim3(kJoinThreads), 0, stream, p, H);
    return launched("attn_decode");
}

size_t decode_bytes(const DecodePlan& plan, int d) { return plan.direct ? 0 : (size_t)plan.grid * (2 * plan.heads_kept * (d + 2) * sizeof(float) + sizeof(int4)); }

// Checks the arguments of attn_decode (those that decode_plan and check_cache leave) and fills in what the kernels get of them, the workspace apart.
int decode_params(const void* Q, int64_t q_request, int64_t q_head, void* O, int64_t o_request, int64_t o_head, int o_dtype, const sawattn_kv_cache* cache,
                  const int32_t* table, int64_t table_stride, int max_pages, const int32_t* lengths, int R, int H, float scale, int window, void* workspace,
                  size_t workspace_bytes, size_t need, const DecodePlan& plan, DecodeParams* out) {
    if (!Q || !O || !table || !lengths || (need && !workspace))
        return fail(SAWATTN_ERR_INVALID_ARG, "Q, O, table, lengths and workspace must be non-null");
    if (cache->k_row > (1 << 26) || cache->v_row > (1 << 26)) return fail(SAWATTN_ERR_UNSUPPORTED, "cache: row strides must be at most 2^26");
    if (((uintptr_t)Q | (uintptr_t)O | (uintptr_t)workspace) & 15u)
        return fail(SAWATTN_ERR_INVALID_ARG, "Q, O and workspace must be 16-byte aligned");
    if (((uintptr_t)table | (uintptr_t)lengths) & 3u) return fail(SAWATTN_ERR_INVALID_ARG, "table and lengths must be 4-byte aligned");
    if (o_dtype != SAWATTN_F16 && o_dtype != SAWATTN_BF16 && o_dtype != SAWATTN_F32)
        return fail(SAWATTN_ERR_INVALID_ARG, "o_dtype must be SAWATTN_F16, SAWATTN_BF16 or SAWATTN_F32");
    if (!std::isfinite(scale)) return fail(SAWATTN_ERR_INVALID_ARG, "scale must be finite");
    if (table_stride < max_pages || (double)table_stride * R >= 1e18)
        return fail(SAWATTN_ERR_INVALID_ARG, "table_stride must be at least max_pages");
    const int d = cache->d;
    if (!good_stride(q_request, R) || !good_stride(q_head, H) || !good_stride(o_request, R) || !good_stride(o_head, H))
        return fail(SAWATTN_ERR_INVALID_ARG, "strides of Q and O must be multiples of 8, not negative");
    if ((R > 1 && o_request < d) || (H > 1 && o_head < d)) return fail(SAWATTN_ERR_INVALID_ARG, "strides of O must be at least d");
    if (workspace_bytes < need)
        return fail(SAWATTN_ERR_INVALID_ARG, "workspace is smaller than attn_decode_workspace_bytes reports");
    const int o_size = o_dtype == SAWATTN_F32 ? 4 : 2;
    auto extent = [](int n, int64_t stride) { return n > 1 ? (unsigned long long)(n - 1) * stride : 0ull; };
    const Range o(O, o_size * (extent(R, o_request) + extent(H, o_head) + d));
    const Range scratch(workspace, need);
    const Range in[] = {
        {Q, 2 * (extent(R, q_request) + extent(H, q_head) + d)},
        {cache->k, 2 * (extent(cache->pages, cache->k_page) + extent(cache->heads, cache->k_head) + extent(cache->page_size, cache->k_row) + d)},
        {cache->v, 2 * (extent(cache->pages, cache->v_page) + extent(cache->heads, cache->v_head) + extent(cache->page_size, cache->v_row) + d)},
        {table, 4 * (extent(R, table_stride) + max_pages)}, {lengths, 4ull * R}};
    for (const Range& i : in)
        if (o.meets(i) || scratch.meets(i)) return fail(SAWATTN_ERR_INVALID_ARG, "O and workspace must not overlap what is read");
    if (o.meets(scratch)) return fail(SAWATTN_ERR_INVALID_ARG, "O must not overlap the workspace");

    *out = DecodeParams{};
    DecodeParams& p = *out;
    p.Q = static_cast<const char*>(Q); p.q_request = 2 * q_request; p.q_head = 2 * q_head;
    p.O = static_cast<char*>(O); p.o_request = o_size * o_request; p.o_head = o_size * o_head; p.o_dtype = o_dtype;
    p.K = static_cast<const char*>(cache->k); p.V = static_cast<const char*>(cache->v);
    p.k_page = 2 * cache->k_page; p.k_head = 2 * cache->k_head; p.k_row = (unsigned)(2 * cache->k_row);
    p.v_page = 2 * cache->v_page; p.v_head = 2 * cache->v_head; p.v_row = (unsigned)(2 * cache->v_row);
    p.table = table; p.table_stride = table_stride; p.lengths = lengths;
    p.c = (float)((double)scale * 1.4426950408889634074);
    p.R = R; p.capacity = max_pages * cache->page_size; p.window = window; p.pages = cache->pages; p.shift = page_shift(cache->page_size);
    p.group = plan.group; p.head_groups = plan.head_groups; p.units = plan.units; p.workgroups = plan.workgroups; p.heads_kept = plan.heads_kept;
    return SAWATTN_OK;
}

// Launches what decode_params has filled in; workspace: of decode_bytes, NULL where that is 0.
int run_decode(DecodeParams& p, const DecodePlan& plan, int H, int d, int dtype, void* workspace, hipStream_t stream) {
    if (workspace) {
        p.parts = static_cast<float*>(workspace);
        p.begun = reinterpret_cast<int4*>(p.parts + (size_t)2 * plan.grid * plan.heads_kept * d);
        p.part_sums = reinterpret_cast<f2*>(p.begun + plan.grid);
    }
    const bool bf = dtype == SAWATTN_BF16;
    if (d == 128) return bf ? launch_decode<128, true>(p, plan, H, stream) : launch_decode<128, false>(p, plan, H, stream);
    return bf ? launch_decode<64, true>(p, plan, H, stream) : launch_decode<64, false>(p, plan, H, stream);
}

}  // namespace sawattn

extern "C" {

int attn_decode_workspace_bytes(const sawattn_kv_cache* cache, int R, int H, int max_pages, size_t* bytes) {
    using namespace sawattn;
    if (!bytes) return fail(SAWATTN_ERR_INVALID_ARG, "bytes must be non-null");
    int rc = check_cache(cache, false);
    if (rc != SAWATTN_OK) return rc;
    DecodePlan plan;
    rc = decode_plan(cache, R, H, max_pages, 0, &plan);
    if (rc != SAWATTN_OK) return rc;
    // Enough for smaller batches too.  The need rises with R and max_pages while units are shared; where there are so many of them that they are not, it is
    // that of the largest batch for which they are.
    const int shared = (int)std::min<long long>(R, (kDecodeUnits - 1) / ((long long)plan.units * plan.head_groups));
    if (plan.direct && shared > 0) {
        rc = decode_plan(cache, shared, H, max_pages, 0, &plan);
        if (rc != SAWATTN_OK) return rc;
    }
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
    if (window < 0) return fail(SAWATTN_ERR_INVALID_ARG, "window must not be negative");
    DecodePlan plan;
    rc = decode_plan(cache, R, H, max_pages, window, &plan);
    if (rc != SAWATTN_OK) return rc;
    const size_t need = decode_bytes(plan, cache->d);
    DecodeParams p;
    rc = decode_params(Q, q_request, q_head, O, o_request, o_head, o_dtype, cache, table, table_stride, max_pages, lengths, R, H, scale, window, workspace,
                       workspace_bytes, need, plan, &p);
    if (rc != SAWATTN_OK) return rc;
    return run_decode(p, plan, H, cache->d, cache->dtype, need ? workspace : nullptr, static_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
