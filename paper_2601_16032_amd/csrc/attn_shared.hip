// attn_decode_shared: attention of one new token per request, for groups of requests that begin with the same rows.
//
//   s_j = scale q . k_j,  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m);  over two sets of rows with (m1, l1, o1) and (m2, l2, o2), o = sum p v:
//   m = max(m1, m2),  O = (exp(m1 - m) o1 + exp(m2 - m) o2) / (exp(m1 - m) l1 + exp(m2 - m) l2)
//
// A prefix unit is a group's common rows in one key/value head, with up to 16 NB of the query heads that look at them (its columns: all query
// heads of that key head of all requests of the group, one request's behind the other's); a tail unit is the rows behind them of one request, with up
// to 16 of its query heads, as in attn_decode.  Tails are bound by memory.  A prefix is read once for all of a unit's columns, 4 d flops
// for each of them per 4 d bytes: from 64 columns on it is the matrix cores' and the vector units' time that counts.
//
// Who does what.  The steps (128 rows) of all prefix units, one behind the other, are dealt out evenly over the workgroups, and so are those of all tail
// units, the other way round.  Every workgroup takes its share of both; of the two workgroups of a compute unit one begins with
// prefixes and one with tails, so that one computes while the other waits for memory.  Of each unit that it ends, begins or goes on
// with it leaves (m, l, o) in the workspace, and a second kernel joins for every row of O what belongs to it.
//
// Within a workgroup it goes as in attn_decode: every wavefront takes tiles of 32 rows of its own, transposed products on 16x16x32 MFMAs, K by way of LDS,
// V in registers.  A prefix tile is loaded once and meets NB blocks of 16 columns.
// The probabilities enter the second product as sums of two 16-bit numbers (SharedPieces), 16 bits of them and more; those of the tails as in attn_decode.
namespace sawattn {

constexpr int kSharedThreads = 64 * kDecodeWaves;
constexpr int kSharedGrid = 512;      // workgroups: two to a compute unit
constexpr int kSharedMostColumns = 64;

struct SharedParams {
    DecodeParams d;           // the query, the cache, the table, as in attn_decode (its workspace is not used)
    const int* offsets;       // [groups + 1]
    const int* shared;        // [groups]
    int groups, H;
    // workspace
    float* prefix_parts;      // [2 * grid][columns of a unit][D]
    f2* prefix_sums;
    float* tail_parts;        // [2 * grid][heads_kept][D]
    f2* tail_sums;
    float* rows[2];           // [R][H][D] of prefix units, of tail units that one workgroup did all of
    f2* row_sums[2];
    int4* requests;           // [R] (first request of the group, rows in common, group, length)
    int2* prefix_records;     // per unit: (first workgroup, last one); first -1: all of it is in `rows`
    int2* tail_records;
};

// Two probabilities as sums of two 16-bit numbers each.  The first is cut off, of the next smaller number in bfloat16, so that something is left; the second is what is
// left, rounded (bfloat16: off by 2^-16 of the probability at most) or cut off (binary16: 2^-21, or 2^-39 of the largest where that is more).
template <bool BF16>
struct SharedPieces {
    static constexpr int kCount = 2;
    unsigned word[kCount];
    __device__ __forceinline__ SharedPieces(float a, float b) {
        if constexpr (BF16) {
            const unsigned x = __builtin_elementwise_sub_sat(__builtin_bit_cast(unsigned, a), 1u), y = __builtin_elementwise_sub_sat(__builtin_bit_cast(unsigned, b), 1u);
            word[0] = __builtin_amdgcn_perm(y, x, 0x07060302u);
            word[1] = narrow<true>(a - __builtin_bit_cast(float, x & 0xffff0000u), b - __builtin_bit_cast(float, y & 0xffff0000u));
        } else {
            word[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(a, b));
            word[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(fmaxf(a - widen<false>(word[0], 0), fminf(a, 0x1p-24f)),
                                                                              fmaxf(b - widen<false>(word[0], 1), fminf(b, 0x1p-24f))));
        }
    }
};

// A wavefront's part of a prefix unit.
template <int D, bool BF16, int NB>
struct PrefixState {
    f4 o[NB][D / 16];        // as DecodeState::o, for each block of 16 columns
    float m[NB], l[NB];

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[b][j] = f4{0.f, 0.f, 0.f, 0.f};
            m[b] = -INFINITY;
            l[b] = 0.f;
        }
    }

    // q: the unit's queries in LDS, operands of (block, 32 elements), 16 bytes to a lane.  All columns see all rows up to u.length.
    __device__ __forceinline__ void add(const DecodeParams& p, const DecodeLane<D>& lane, const DecodeUnit& u, LDS_PTR(const u4) q, int blocks, const DecodePages& pages,
                                        int tile, LDS_PTR(char) lds) {
        using L = DecodeLane<D>;
        const int mask = (1 << p.shift) - 1, key0 = tile * kDecodeTile;
        const bool edge = key0 + kDecodeTile > u.length;
        bool bad[2];
        unsigned v[8][D / 32];
#pragma unroll
        for (int half = 0; half < 2; ++half) bad[half] = (unsigned)pages.half[half] >= (unsigned)p.pages;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int page = bad[half] ? 0 : pages.half[half], row = (key0 + half * 16) & mask;
            const char* k = u.K + page * p.k_page + (long long)row * p.k_row;
#pragma unroll
            for (int i = 0; i < L::kLoads / 2; ++i)
                load_to_lds_16B(k + (long long)i * L::kRowsPerLoad * p.k_row, lane.k_from(i), (unsigned)(uintptr_t)lds + (half * (L::kLoads / 2) + i) * 1024);
        }
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int page = bad[half] ? 0 : pages.half[half], row = (key0 + half * 16) & mask;
            const char* from = u.V + page * p.v_page + (long long)row * p.v_row;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                typedef unsigned words __attribute__((ext_vector_type(D / 32)));
                const words w = *reinterpret_cast<const words*>(from + (long long)i * 4 * p.v_row + lane.v_from);
#pragma unroll
                for (int x = 0; x < D / 32; ++x) v[half * 4 + i][x] = w[x];
            }
        }
        asm volatile("s_waitcnt vmcnt(8)" ::: "memory");      // K has landed, V is on its way
        f4 s[NB][2];
#pragma unroll
        for (int b = 0; b < NB; ++b) s[b][0] = s[b][1] = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < D / 32; ++x) {
            u4 k[2];
#pragma unroll
            for (int half = 0; half < 2; ++half) k[half] = *(LDS_PTR(const u4))(lds + lane.k_operand(x) + half * 16 * L::kRowBytes);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (b < blocks) {
                    const u4 operand = q[(b * (D / 32) + x) * 64];
#pragma unroll
                    for (int half = 0; half < 2; ++half) s[b][half] = decode_mfma<BF16>(k[half], operand, s[b][half]);
                }
            }
        }
#pragma unroll
        for (int b = 0; b < NB; ++b)
            if (b < blocks) {
#pragma unroll
                for (int half = 0; half < 2; ++half) s[b][half] *= p.c;
            }
        if (edge || bad[0] || bad[1]) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool seen = key0 + 4 * i + lane.g < u.length;
#pragma unroll
                for (int b = 0; b < NB; ++b) s[b][i / 4][i % 4] = !seen ? -INFINITY : bad[i / 4] ? __builtin_nanf("") : s[b][i / 4][i % 4];
                if (!seen) {      // whatever the row holds, it takes no part: 0 * NaN would
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) v[i][x] = 0;
                }
            }
        }
        using Pieces = SharedPieces<BF16>;
        u4 piece[NB][Pieces::kCount];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            if (b >= blocks) continue;
            float most = fmaxf(fmaxf(fmaxf(s[b][0][0], s[b][0][1]), fmaxf(s[b][0][2], s[b][0][3])), fmaxf(fmaxf(s[b][1][0], s[b][1][1]), fmaxf(s[b][1][2], s[b][1][3])));
            most = head_max(most);
            if (__any(most > m[b])) {
                const float next = fmaxf(m[b], most), fade = next == -INFINITY ? 1.f : fast_exp2(m[b] - next);
                m[b] = next;
                l[b] *= fade;
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[b][j] *= fade;
            }
            const float reference = (m[b] == -INFINITY ? 0.f : m[b]) - (BF16 ? 0.f : 15.f);
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float x = fast_exp2(s[b][w / 2][w % 2 * 2] - reference), y = fast_exp2(s[b][w / 2][w % 2 * 2 + 1] - reference);
                l[b] += x + y;
                const Pieces pieces(x, y);
#pragma unroll
                for (int i = 0; i < Pieces::kCount; ++i) piece[b][i][w] = pieces.word[i];
            }
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            u4 a;      // element j of the lane's pieces of its eight rows
#pragma unroll
            for (int w = 0; w < 4; ++w) a[w] = __builtin_amdgcn_perm(v[2 * w + 1][j / 2], v[2 * w][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (b >= blocks) continue;
#pragma unroll
                for (int i = 0; i < Pieces::kCount; ++i) o[b][j] = decode_mfma<BF16>(a, piece[b][i], o[b][j]);
            }
        }
    }
};

// The wavefronts' parts of up to 16 columns, added up; store(column, element / 4, m, l, o) gets the sums.
template <int D, typename STORE>
__device__ __forceinline__ void join_waves(char (*area)[kDecodeHeads * (D + 4) * 4], float (*m_of)[kDecodeHeads], float (*l_of)[kDecodeHeads], const f4 (&state)[D / 16],
                                           float state_m, float state_l, int wave, int columns, STORE&& store) {
    constexpr int kPitch = D + 4;
    const float sum = head_sum(state_l);
    const int now = lane_now(), c = now & 15, g = now >> 4;
    if (g == 0) {
        m_of[wave][c] = state_m;
        l_of[wave][c] = sum;
    }
    float* o = reinterpret_cast<float*>(area[wave]) + c * kPitch;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < D / 16; j += 4)
            *reinterpret_cast<f4*>(o + (4 * g + i) * (D / 16) + j) = f4{state[j][i], state[j + 1][i], state[j + 2][i], state[j + 3][i]};
    __syncthreads();
    for (int e = wave * 64 + now; e < columns * (D / 4); e += kSharedThreads) {
        const int column = e / (D / 4), at4 = e % (D / 4) * 4;
        float m = m_of[0][column];
#pragma unroll
        for (int w = 1; w < kDecodeWaves; ++w) m = fmaxf(m, m_of[w][column]);
        const float reference = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        f4 x = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kDecodeWaves; ++w) {
            const float f = fast_exp2(m_of[w][column] - reference);
            l += f * l_of[w][column];
            x += f * *reinterpret_cast<const f4*>(reinterpret_cast<const float*>(area[w]) + column * kPitch + at4);
        }
        store(column, at4, m, l, x);
    }
    __syncthreads();
}

// Sum of x over the threads in front of this one, and over all of the workgroup.
__device__ __forceinline__ int shared_before(int x, int* of_wave, int& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, upto = lanes_upto(x);
    if (lane == 63) of_wave[wave] = upto;
    __syncthreads();
    int before = upto - x;
    all = 0;
#pragma unroll
    for (int w = 0; w < kDecodeWaves; ++w) {
        if (w < wave) before += of_wave[w];
        all += of_wave[w];
    }
    return before;
}

// What the workgroup knows of the groups, in LDS: where they begin (groups + 1 of them), and the rows they have in common.
struct SharedGroups {
    int* offsets;
    int* common;
    int* lead;
    int groups;
    __device__ __forceinline__ int of_request(int r) const {      // the request's group, or -1
        if (r < offsets[0]) return -1;
        int low = 0, high = groups;
        while (low < high) {      // the first group that begins behind it
            const int mid = (low + high) >> 1;
            if (offsets[mid + 1] > r) high = mid; else low = mid + 1;
        }
        return low < groups && offsets[low] <= r ? low : -1;
    }
};

struct SharedStart {      // of a workgroup's share, found by one of its threads
    int item, inside;
};

template <int D, bool BF16, int NB>
__global__ __launch_bounds__(kSharedThreads, 2) void decode_shared_kernel(SharedParams p) {
    constexpr int kPitch = D + 4, kArea = kDecodeHeads * kPitch * 4, kColumns = 16 * NB;
    __shared__ __align__(16) char area[kDecodeWaves][kArea];
    __shared__ __align__(16) u4 queries[NB * (D / 32) * 64];
    __shared__ float m_of[kDecodeWaves][kDecodeHeads], l_of[kDecodeWaves][kDecodeHeads];
    __shared__ int of_wave[2][kDecodeWaves];
    __shared__ SharedStart start[2];
    __shared__ int falls;
    extern __shared__ int lists[];      // offsets [groups + 1], rows in common [groups], first request that is not empty [groups]
    const DecodeParams& d = p.d;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const SharedGroups in = {lists, lists + p.groups + 1, lists + 2 * p.groups + 1, p.groups};

    // ---- the groups
    if (tid == 0) falls = 0;
    for (int g = tid; g <= p.groups; g += kSharedThreads) in.offsets[g] = min(max(p.offsets[g], 0), d.R);
    for (int g = tid; g < p.groups; g += kSharedThreads) {
        in.common[g] = 0x7fffffff;
        in.lead[g] = d.R;
    }
    auto length_of = [&](int r) { return min(max(d.lengths[r], 0), d.capacity); };
    __syncthreads();
    for (int g = tid; g < p.groups; g += kSharedThreads)
        if (in.offsets[g] > in.offsets[g + 1]) falls = 1;
    for (int r = tid; r < d.R; r += kSharedThreads) {
        const int length = length_of(r), g = in.of_request(r);
        if (length && g >= 0) {
            atomicMin(&in.common[g], length);
            atomicMin(&in.lead[g], r);
        }
    }
    __syncthreads();
    auto blocks_of = [&](int g) { return ((in.offsets[g + 1] - in.offsets[g]) * d.group + kColumns - 1) / kColumns; };
    auto prefix_steps = [&](int g) { return (in.common[g] + kDecodeStep - 1) / kDecodeStep; };
    const int each_group = (p.groups + kSharedThreads - 1) / kSharedThreads, g0 = tid * each_group;
    int mine = 0;
    for (int i = 0; i < each_group; ++i) {
        const int g = g0 + i;
        if (g >= p.groups) break;
        const int size = in.offsets[g + 1] - in.offsets[g], common = in.lead[g] < d.R && size > 1 && !falls ? max(min(in.common[g], p.shared[g]), 0) >> d.shift << d.shift : 0;
        in.common[g] = common;
        if (common) mine += prefix_steps(g) * blocks_of(g) * d.units;
    }
    int total_prefix, total_tail;
    int before_prefix = shared_before(mine, of_wave[0], total_prefix);      // (a barrier in it: what the groups have in common is there)
    const int mine_prefix = mine;
    // ---- the requests
    auto tail_from = [&](int g) { return g >= 0 ? in.common[g] : 0; };
    auto tail_steps = [&](int length, int from) { return length > from ? (length - 1) / kDecodeStep - from / kDecodeStep + 1 : 0; };
    const int each = (d.R + kSharedThreads - 1) / kSharedThreads, r0 = tid * each;
    const int units = d.units * d.head_groups;
    mine = 0;
    for (int i = 0; i < each; ++i) {
        const int r = r0 + i;
        if (r >= d.R) break;
        const int length = length_of(r), g = in.of_request(r), from = tail_from(g);
        mine += tail_steps(length, from) * units;
        if (blockIdx.x == 0) p.requests[r] = int4{g >= 0 ? in.offsets[g] : r, from, max(g, 0), length};
    }
    int before_tail = shared_before(mine, of_wave[1], total_tail);
    const int grid = gridDim.x, block = blockIdx.x;
    const int share_prefix = (int)(((unsigned)total_prefix + grid - 1) / (unsigned)grid), share_tail = (int)(((unsigned)total_tail + grid - 1) / (unsigned)grid);
    // Workgroups go round the XCDs; those of one XCD take neighbouring shares, which read the same rows where a group has several units.
    const int wp = share_prefix > 1 ? block % 8 * (grid / 8) + block / 8 : block, wt = grid - 1 - block;
    const int at_prefix = wp * share_prefix, at_tail = wt * share_tail;      // (below the totals and twice the grid)
    int left_prefix = min(share_prefix, total_prefix - at_prefix), left_tail = min(share_tail, total_tail - at_tail);
    if (left_prefix > 0 && at_prefix >= before_prefix && at_prefix < before_prefix + mine_prefix) {
        int g = g0;
        for (;; ++g) {
            const int steps = in.common[g] ? prefix_steps(g) * blocks_of(g) * d.units : 0;
            if (at_prefix < before_prefix + steps) break;
            before_prefix += steps;
        }
        start[0] = SharedStart{g, at_prefix - before_prefix};
    }
    if (left_tail > 0 && at_tail >= before_tail && at_tail < before_tail + mine) {
        int r = r0;
        for (; r < min(r0 + each, d.R) - 1; ++r) {      // (the last one if the lengths have changed meanwhile)
            const int steps = tail_steps(length_of(r), tail_from(in.of_request(r))) * units;
            if (at_tail < before_tail + steps) break;
            before_tail += steps;
        }
        start[1] = SharedStart{r, at_tail - before_tail};
    }
    __syncthreads();

    const DecodeLane<D> lane(d, tid & 63);
    auto prefixes = [&]() {
        if (left_prefix <= 0) return;
        int g = __builtin_amdgcn_readfirstlane(start[0].item);
        const int inside = __builtin_amdgcn_readfirstlane(start[0].inside);
        int steps = __builtin_amdgcn_readfirstlane(prefix_steps(g)), blocks = __builtin_amdgcn_readfirstlane(blocks_of(g));
        int t0 = (unsigned)inside % (unsigned)steps, part = (unsigned)inside / (unsigned)steps;      // part: unit * blocks + block
        do {
            const int t1 = min(steps, t0 + left_prefix), unit = (unsigned)part / (unsigned)blocks, column0 = (part - unit * blocks) * kColumns;
            const int begin = __builtin_amdgcn_readfirstlane(in.offsets[g]), columns = min((__builtin_amdgcn_readfirstlane(in.offsets[g + 1]) - begin) * d.group - column0, kColumns);
            auto row_of = [&](int column, int& r) {      // request and query head of a column
                const int at = column0 + column, i = (unsigned)at / (unsigned)d.group;
                r = begin + i;
                return unit * d.group + at - i * d.group;
            };
            for (int e = tid; e < NB * (D / 32) * 64; e += kSharedThreads) {
                const int column = e / (64 * (D / 32)) * 16 + e % 16, from = e / 64 % (D / 32) * 64 + e % 64 / 16 * 16;
                u4 x = {0, 0, 0, 0};
                if (column < columns) {
                    int r;
                    const int head = row_of(column, r);
                    x = *reinterpret_cast<const u4*>(d.Q + r * d.q_request + head * d.q_head + from);
                }
                queries[e] = x;
            }
            __syncthreads();
            const int length = __builtin_amdgcn_readfirstlane(in.common[g]), lead = __builtin_amdgcn_readfirstlane(in.lead[g]);
            const DecodeUnit u = {d.K + unit * d.k_head, d.V + unit * d.v_head,
                                  (const __attribute__((address_space(4))) int*)(uintptr_t)(d.table + lead * d.table_stride), 0, length};
            PrefixState<D, BF16, NB> state;
            state.clear();
            int tile = t0 * kDecodeWaves + wave;
            const int tiles = min(t1 * kDecodeWaves, (length + kDecodeTile - 1) / kDecodeTile), blocks16 = (columns + 15) / 16;
            if (tile < tiles) {
                DecodePages pages(d, u, tile);
                do {
                    const int next = tile + kDecodeWaves;
                    const DecodePages ahead(d, u, next);
                    state.add(d, lane, u, (LDS_PTR(const u4))queries + (tid & 63), blocks16, pages, tile, (LDS_PTR(char))area[wave]);
                    pages = ahead;
                    tile = next;
                } while (tile < tiles);
            }
            const bool whole = t0 == 0 && t1 == steps;
            const long long place = 2 * wp + (t0 == 0 ? 1 : 0);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                if (b >= blocks16) continue;
                join_waves<D>(area, m_of, l_of, state.o[b], state.m[b], state.l[b], wave, min(16, columns - 16 * b), [&](int column, int at4, float m, float l, f4 o) {
                    long long row = place * kColumns + b * 16 + column;
                    float* to = p.prefix_parts;
                    f2* sums = p.prefix_sums;
                    if (whole) {
                        int r;
                        const int head = row_of(b * 16 + column, r);
                        row = (long long)r * p.H + head;
                        to = p.rows[0];
                        sums = p.row_sums[0];
                    }
                    *reinterpret_cast<f4*>(to + row * D + at4) = o;
                    if (at4 == 0) sums[row] = f2{m, l};
                });
            }
            if (t0 == 0 && tid == 0) {
                const long long record = ((long long)begin * d.group / kColumns + g + (part - unit * blocks)) * d.units + unit;
                p.prefix_records[record] = whole ? int2{-1, 0} : int2{wp, min(wp + (steps - t1 + share_prefix - 1) / share_prefix, grid - 1)};
            }
            left_prefix -= t1 - t0;
            t0 = 0;
            if (left_prefix > 0 && ++part == blocks * d.units) {
                part = 0;
                do {
                    if (++g >= p.groups) return;      // (not reached)
                } while (__builtin_amdgcn_readfirstlane(in.common[g]) == 0);
                steps = __builtin_amdgcn_readfirstlane(prefix_steps(g));
                blocks = __builtin_amdgcn_readfirstlane(blocks_of(g));
            }
        } while (left_prefix > 0);
    };
    auto tails = [&]() {
        if (left_tail <= 0) return;
        int r = __builtin_amdgcn_readfirstlane(start[1].item);
        const int inside = __builtin_amdgcn_readfirstlane(start[1].inside);
        int length = __builtin_amdgcn_readfirstlane(length_of(r)), from = __builtin_amdgcn_readfirstlane(tail_from(in.of_request(r))), steps = max(tail_steps(length, from), 1);
        int t0 = (unsigned)inside % (unsigned)steps, part = min((int)((unsigned)inside / (unsigned)steps), units - 1);      // part: unit * head groups + head group
        do {
            const int t1 = min(steps, t0 + left_tail), unit = (unsigned)part / (unsigned)d.head_groups, head_group = part - unit * d.head_groups;
            const int head0 = head_group * kDecodeHeads, heads = min(kDecodeHeads, d.group - head0);
            const char* q_row = d.Q + r * d.q_request + (long long)(unit * d.group + head0) * d.q_head;
            u4 q[D / 32];
#pragma unroll
            for (int x = 0; x < D / 32; ++x)
                q[x] = lane.c < heads ? *reinterpret_cast<const u4*>(q_row + lane.c * d.q_head + x * 64 + lane.g * 16) : u4{0, 0, 0, 0};
            const DecodeUnit u = {d.K + unit * d.k_head, d.V + unit * d.v_head,
                                  (const __attribute__((address_space(4))) int*)(uintptr_t)(d.table + r * d.table_stride), from, length};
            DecodeState<D, BF16> state;
            state.clear();
            const int first = from / kDecodeStep;
            int tile = (first + t0) * kDecodeWaves + wave;
            const int tiles = min((first + t1) * kDecodeWaves, (length + kDecodeTile - 1) / kDecodeTile);
            if ((tile + 1) * kDecodeTile <= from) tile += kDecodeWaves;
            if (tile < tiles) {
                DecodePages pages(d, u, tile);
                do {
                    const int next = tile + kDecodeWaves;
                    const DecodePages ahead(d, u, next);
                    state.template add<false>(d, lane, u, q, pages, tile, (LDS_PTR(char))area[wave]);
                    pages = ahead;
                    tile = next;
                } while (tile < tiles);
            }
            const bool whole = t0 == 0 && t1 == steps;
            const long long place = 2 * wt + (t0 == 0 ? 1 : 0);
            join_waves<D>(area, m_of, l_of, state.o, state.m, state.l, wave, heads, [&](int column, int at4, float m, float l, f4 o) {
                const long long row = whole ? (long long)r * p.H + unit * d.group + head0 + column : place * d.heads_kept + column;
                *reinterpret_cast<f4*>((whole ? p.rows[1] : p.tail_parts) + row * D + at4) = o;
                if (at4 == 0) (whole ? p.row_sums[1] : p.tail_sums)[row] = f2{m, l};
            });
            if (t0 == 0 && tid == 0)
                p.tail_records[(long long)r * units + part] = whole ? int2{-1, 0} : int2{wt, min(wt + (steps - t1 + share_tail - 1) / share_tail, grid - 1)};
            left_tail -= t1 - t0;
            t0 = 0;
            if (left_tail > 0 && ++part == units) {
                part = 0;
                do {
                    if (++r >= d.R) return;      // (not reached unless the lengths have changed meanwhile)
                    length = __builtin_amdgcn_readfirstlane(length_of(r));
                    from = __builtin_amdgcn_readfirstlane(tail_from(in.of_request(r)));
                    steps = tail_steps(length, from);
                } while (steps == 0);
            }
        } while (left_tail > 0);
    };
    // (blocks go round the XCDs and, in them, round the 32 compute units)
    if (block / 256 % 2 == 0) {
        prefixes();
        tails();
    } else {
        tails();
        prefixes();
    }
}

// Joins for every row of O the parts of its prefix unit and of its tail unit.  A row is D / 4 threads'; GROUPS of them go over every GROUPS-th part.
constexpr int kSharedJoinThreads = 256, kSharedJoinAhead = 4;

template <int D, int GROUPS>
__global__ __launch_bounds__(kSharedJoinThreads) void decode_shared_join_kernel(SharedParams p, int columns, int grid) {
    constexpr int kAcross = D / 4, kRows = kSharedJoinThreads / (kAcross * GROUPS);
    __shared__ f4 o_of[GROUPS][kRows][kAcross];
    __shared__ f2 sums_of[GROUPS][kRows];
    const DecodeParams& d = p.d;
    const int tid = threadIdx.x, a = tid % kAcross, of_row = tid / kAcross % kRows, group = tid / (kAcross * kRows);
    const long long row = (long long)blockIdx.x * kRows + of_row;
    const bool there = row < (long long)d.R * p.H;
    const int r = there ? (int)((unsigned)row / (unsigned)p.H) : 0, head = there ? (int)(row - (long long)r * p.H) : 0;
    const int4 request = p.requests[r];      // (first request of the group, rows in common, group, length)
    const int unit = (unsigned)head / (unsigned)d.group, in_unit = head - unit * d.group;
    float m = -INFINITY, l = 0.f;
    f4 o = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](int2 record, const float* parts, const f2* sums, int kept, int column, const float* rows, const f2* row_sums) {
        const bool whole = record.x < 0;
        const int first = whole ? 0 : max(record.x, 0), last = whole ? 0 : min(record.y, grid - 1);
        for (int w = first + group; w <= last; w += GROUPS * kSharedJoinAhead) {
            f2 of[kSharedJoinAhead];
            f4 part[kSharedJoinAhead];
            float next = m;
#pragma unroll
            for (int i = 0; i < kSharedJoinAhead; ++i) {
                const int at = min(w + i * GROUPS, last);
                const long long place = whole ? row : (long long)(2 * at + (at == first ? 1 : 0)) * kept + column;
                of[i] = (whole ? row_sums : sums)[place];
                part[i] = *reinterpret_cast<const f4*>((whole ? rows : parts) + place * D + a * 4);
            }
#pragma unroll
            for (int i = 0; i < kSharedJoinAhead; ++i) next = fmaxf(next, of[i][0]);
            const float reference = next == -INFINITY ? 0.f : next, fade = fast_exp2(m - reference);
            l *= fade;
            o *= fade;
#pragma unroll
            for (int i = 0; i < kSharedJoinAhead; ++i)
                if (w + i * GROUPS <= last) {
                    const float f = fast_exp2(of[i][0] - reference);
                    l += of[i][1] * f;
                    o += part[i] * f;
                }
            m = next;
        }
    };
    const bool seen = there && request.w > 0, behind = seen && request.w > request.y, common = seen && request.y > 0;
    const int at = (r - request.x) * d.group + in_unit, block = (unsigned)at / (unsigned)columns, head_group = in_unit / kDecodeHeads;
    int2 prefix = {0, -1}, tail = {0, -1};
    if (common) prefix = p.prefix_records[((long long)request.x * d.group / columns + request.z + block) * d.units + unit];
    if (behind) tail = p.tail_records[((long long)r * d.units + unit) * d.head_groups + head_group];
    if (common) add(prefix, p.prefix_parts, p.prefix_sums, columns, at - block * columns, p.rows[0], p.row_sums[0]);
    if (behind) add(tail, p.tail_parts, p.tail_sums, d.heads_kept, in_unit - head_group * kDecodeHeads, p.rows[1], p.row_sums[1]);
    if constexpr (GROUPS > 1) {
        o_of[group][of_row][a] = o;
        if (a == 0) sums_of[group][of_row] = f2{m, l};
        __syncthreads();
        if (group != 0) return;
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) m = fmaxf(m, sums_of[i][of_row][0]);
        const float reference = m == -INFINITY ? 0.f : m;
        l = 0.f;
        o = f4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) {
            const float f = fast_exp2(sums_of[i][of_row][0] - reference);
            l += f * sums_of[i][of_row][1];
            o += f * o_of[i][of_row][a];
        }
    }
    if (!there) return;
    const int o_size = d.o_dtype == SAWATTN_F32 ? 4 : 2;
    store_o(d.O + r * d.o_request + head * d.o_head + a * 4 * o_size, d.o_dtype, seen ? o / l : f4{0.f, 0.f, 0.f, 0.f});
}

// The workspace, in bytes from the front: for the widest units, whichever a call takes.
struct SharedWorkspace {
    size_t prefix_sums, tail_parts, tail_sums, rows[2], row_sums[2], requests, prefix_records, tail_records, all;
    SharedWorkspace(const DecodePlan& plan, int R, int H, int groups, int d) {
        const size_t places = 2 * kSharedGrid, columns = std::min<long long>(kSharedMostColumns, ((long long)R * plan.group + 15) / 16 * 16), n = (size_t)R * H;
        size_t at = places * columns * d * 4;
        auto next = [&](size_t& where, size_t bytes) { where = at; at += (bytes + 15) / 16 * 16; };
        next(prefix_sums, places * columns * 8);
        next(tail_parts, places * plan.heads_kept * d * 4);
        next(tail_sums, places * plan.heads_kept * 8);
        for (int i = 0; i < 2; ++i) next(rows[i], n * d * 4);
        for (int i = 0; i < 2; ++i) next(row_sums[i], n * 8);
        next(requests, 16 * (size_t)R);
        next(prefix_records, 8 * ((size_t)R * plan.group / 16 + groups + 1) * plan.units);
        next(tail_records, 8 * (size_t)R * plan.units * plan.head_groups);
        all = at;
    }
};

int shared_plan(const sawattn_kv_cache* cache, int R, int H, int groups, int max_pages, DecodePlan* plan) {
    const int rc = decode_plan(cache, R, H, max_pages, 0, plan);
    if (rc != SAWATTN_OK) return rc;
    if (groups <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "groups must be positive");
    if (R > SAWATTN_MOST_REQUESTS || groups > SAWATTN_MOST_REQUESTS) return fail(SAWATTN_ERR_UNSUPPORTED, "more requests or groups than SAWATTN_MOST_REQUESTS");
    const double steps = ((double)max_pages * cache->page_size + kDecodeStep - 1) / kDecodeStep;
    if (steps * R * H >= 2147483648.0 - 4.0 * kSharedGrid) return fail(SAWATTN_ERR_INVALID_ARG, "R*H*ceil(max_pages*page_size/128) must be below 2^31 - 2048");
    return SAWATTN_OK;
}

template <int D, bool BF16>
int launch_shared(const SharedParams& p, int grid, hipStream_t stream) {
    // As many blocks of 16 columns as the groups fill if they are of one size: a unit computes the ones it has.
    const int mean = (int)(((long long)p.d.R * p.d.group + p.groups - 1) / p.groups), blocks = mean > 32 ? 4 : mean > 16 ? 2 : 1;
    const size_t lists = sizeof(int) * (3 * (size_t)p.groups + 1);
    if (blocks == 4) hipLaunchKernelGGL((decode_shared_kernel<D, BF16, 4>), dim3(grid), dim3(kSharedThreads), lists, stream, p);
    else if (blocks == 2) hipLaunchKernelGGL((decode_shared_kernel<D, BF16, 2>), dim3(grid), dim3(kSharedThreads), lists, stream, p);
    else hipLaunchKernelGGL((decode_shared_kernel<D, BF16, 1>), dim3(grid), dim3(kSharedThreads), lists, stream, p);
    const int rc = launched("attn_decode_shared");
    if (rc != SAWATTN_OK) return rc;
    const int rows = p.d.R * p.H;
    constexpr int kAcross = D / 4, kRows4 = kSharedJoinThreads / (4 * kAcross), kRows1 = kSharedJoinThreads / kAcross;
    if (rows <= 2048) hipLaunchKernelGGL((decode_shared_join_kernel<D, 4>), dim3((rows + kRows4 - 1) / kRows4), dim3(kSharedJoinThreads), 0, stream, p, 16 * blocks, grid);
    else hipLaunchKernelGGL((decode_shared_join_kernel<D, 1>), dim3((rows + kRows1 - 1) / kRows1), dim3(kSharedJoinThreads), 0, stream, p, 16 * blocks, grid);
    return launched("attn_decode_shared");
}

}  // namespace sawattn

extern "C" {

int attn_decode_shared_workspace_bytes(const sawattn_kv_cache* cache, int R, int H, int groups, int max_pages, size_t* bytes) {
    using namespace sawattn;
    if (!bytes) return fail(SAWATTN_ERR_INVALID_ARG, "bytes must be non-null");
    int rc = check_cache(cache, false);
    if (rc != SAWATTN_OK) return rc;
    DecodePlan plan;
    rc = shared_plan(cache, R, H, groups, max_pages, &plan);
    if (rc != SAWATTN_OK) return rc;
    *bytes = SharedWorkspace(plan, R, H, groups, cache->d).all;
    return SAWATTN_OK;
}

int attn_decode_shared(const void* Q, int64_t q_request, int64_t q_head, void* O, int64_t o_request, int64_t o_head, int o_dtype,
                       const sawattn_kv_cache* cache, const int32_t* table, int64_t table_stride, int max_pages, const int32_t* lengths,
                       const int32_t* group_offsets, const int32_t* shared, int groups, int R, int H, float scale, void* workspace,
                       size_t workspace_bytes, void* hip_stream) {
    using namespace sawattn;
    int rc = check_cache(cache, true);
    if (rc != SAWATTN_OK) return rc;
    DecodePlan plan;
    rc = shared_plan(cache, R, H, groups, max_pages, &plan);
    if (rc != SAWATTN_OK) return rc;
    const int d = cache->d;
    const SharedWorkspace at(plan, R, H, groups, d);
    if (!Q || !O || !table || !lengths || !group_offsets || !shared || !workspace)
        return fail(SAWATTN_ERR_INVALID_ARG, "Q, O, table, lengths, group_offsets, shared and workspace must be non-null");
    if (((uintptr_t)group_offsets | (uintptr_t)shared) & 3u) return fail(SAWATTN_ERR_INVALID_ARG, "group_offsets and shared must be 4-byte aligned");
    if (workspace_bytes < at.all) return fail(SAWATTN_ERR_INVALID_ARG, "workspace is smaller than attn_decode_shared_workspace_bytes reports");
    SharedParams p{};
    rc = decode_params(Q, q_request, q_head, O, o_request, o_head, o_dtype, cache, table, table_stride, max_pages, lengths, R, H, scale, 0, workspace, workspace_bytes, at.all,
                       plan, &p.d);
    if (rc != SAWATTN_OK) return rc;
    auto extent = [](int n, int64_t stride) { return n > 1 ? (unsigned long long)(n - 1) * stride : 0ull; };
    const Range o(O, (o_dtype == SAWATTN_F32 ? 4 : 2) * (extent(R, o_request) + extent(H, o_head) + d)), scratch(workspace, at.all);
    for (const Range& i : {Range(group_offsets, 4ull * (groups + 1)), Range(shared, 4ull * groups)})
        if (o.meets(i) || scratch.meets(i)) return fail(SAWATTN_ERR_INVALID_ARG, "O and workspace must not overlap what is read");
    p.offsets = group_offsets; p.shared = shared; p.groups = groups; p.H = H;
    char* const w = static_cast<char*>(workspace);
    p.prefix_parts = reinterpret_cast<float*>(w); p.prefix_sums = reinterpret_cast<f2*>(w + at.prefix_sums);
    p.tail_parts = reinterpret_cast<float*>(w + at.tail_parts); p.tail_sums = reinterpret_cast<f2*>(w + at.tail_sums);
    for (int i = 0; i < 2; ++i) {
        p.rows[i] = reinterpret_cast<float*>(w + at.rows[i]);
        p.row_sums[i] = reinterpret_cast<f2*>(w + at.row_sums[i]);
    }
    p.requests = reinterpret_cast<int4*>(w + at.requests);
    p.prefix_records = reinterpret_cast<int2*>(w + at.prefix_records);
    p.tail_records = reinterpret_cast<int2*>(w + at.tail_records);
    // as many workgroups as there can be steps, in eights
    const double most = ((double)p.d.capacity + kDecodeStep - 1) / kDecodeStep * R * plan.units * plan.head_groups;
    const int grid = (int)std::min<double>(kSharedGrid, std::ceil(most / 8) * 8);
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const bool bf = cache->dtype == SAWATTN_BF16;
    if (d == 128) return bf ? launch_shared<128, true>(p, grid, stream) : launch_shared<128, false>(p, grid, stream);
    return bf ? launch_shared<64, true>(p, grid, stream) : launch_shared<64, false>(p, grid, stream);
}

}  // extern "C"
