// attn_decode_shared: attention of one new token per request, for groups of requests that begin with the same rows.
//
//   s_j = scale q . k_j,  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m);  over two sets of rows with (m1, l1, o1) and (m2, l2, o2), o = sum p v:
//   m = max(m1, m2),  O = (exp(m1 - m) o1 + exp(m2 - m) o2) / (exp(m1 - m) l1 + exp(m2 - m) l2)
//
// A prefix unit is a group's common rows in one key/value head, with up to 128 of the query heads that look at them (its columns: all query
// heads of that key head of all requests of the group, one request's behind the other's); a tail unit is the rows behind them of one request, with up
// to 16 of its query heads, as in attn_decode.  Tails are bound by memory.  A prefix is read once for a unit's columns, 6 d operations of the matrix cores
// (below) for each of them per 4 d bytes: from 64 columns on it is the matrix cores' and the vector units' time that counts.
//
// Who does what.  The steps (128 rows) of all prefix units, one behind the other, are dealt out evenly over workgroups, and the tiles (32 rows) of all tail
// units, the other way round, over wavefronts.
//   Much to do: every workgroup takes its share of both, and of the two workgroups of a compute unit one begins with prefixes and one with tails, so that one
//   computes while the other waits for memory.
//   Little to do: a workgroup takes one kind only, where that ends sooner; what counts then are the steps from one address to the next, a microsecond each.
// Of each unit that a workgroup ends, begins or goes on with it leaves (m, l, o) in the workspace, and a second kernel joins for every row of O what belongs to it.
// (The lists of groups and requests lie in LDS beside the tiles.  At d = 128 two workgroups fit on a compute unit up to 3 groups + requests of about 3900, then
// one: the second half of the grid begins when the first has ended.)
//
// Products run on 16x16x32 MFMAs, transposed: S^T = K Q^T, O^T = V^T P^T.
//   Up to 32 columns (RowsState), and tails: rows from memory straight into the operands' registers.
//   More: tiles of 64 rows through LDS that the four wavefronts share, 32 columns each (WideState).
// Which it is goes by the unit, so groups of any sizes stand in one call.
//
// The probabilities enter the second product as sums of two 16-bit numbers (SharedPieces), 16 bits of them: one would be off by as much as the
// rounding of O to 16 bits, three, as in attn_decode, would take a third more of the matrix cores.  MFMA phases have precedence over other wavefronts' work.
//
// Measured, 32 + 2 x 8 heads of 128, us:
//   256 requests behind 32768 rows, tails up to 2000    256 (prefixes alone 190, tails alone 105): 0.87 PFLOP/s of MFMAs, 40 % of the rate at the 2.1 GHz that the chip
//                                                       then holds; prefixes alone 1.08, a large product 1.28
//   their prefixes, 32 columns at a time                242 instead of 190 (64 requests behind 8192 rows: 31 and 30)
//   their prefixes, without precedence                  210, with it 200 (before other steps that led to 190)
//   their prefixes, exponentials of 32 rows between the MFMAs of those before and behind them   209 (178 with nothing but its MFMAs and what feeds them)
//   256 requests behind 16384 rows and 256 of their own   311; 522 with units as wide as the groups' mean
//   kernels of their own for calls of 16 or 32 columns at most   1 to 2 % less
//   4096 requests, 1024 groups of 4 behind 1024 rows, 8 + 2 x 2 heads   436 (attn_decode 713); 960 in 240 groups 80 (168)
namespace sawattn {

constexpr int kSharedThreads = 64 * kDecodeWaves;
constexpr int kSharedGrid = 512;      // workgroups: two to a compute unit
constexpr int kSharedColumns = 128;   // of a prefix unit at most
// Bytes of K and V, every request's counted, with the tables full, up to which they are read request by request all the same, by attn_decode's kernels; more where these
// need one launch.  The two here take 12 us at least.  32 + 2 x 8 heads of 128, requests x rows in common + own: 4 x 2000 + 100, 35 MB: 14.2 us, attn_decode 12.1; 8 x 2000 + 100, 69 MB: 14.8
// and 16.9; in one launch (the caches serve most of what is read again) 64 x 500 + 100, 159 MB: 20.7 and 11.3.
constexpr long long kSharedFew = 48LL << 20, kSharedFewDirect = 192LL << 20;
// Smaller factors of the scores than this, 0 among them, are attn_decode's kernels': the ones here mask a score by -inf before they multiply it, and divide by the factor.
constexpr float kSharedLeastFactor = 1e-30f;

struct SharedParams {
    DecodeParams d;           // the query, the cache, the table, as in attn_decode (its workspace is not used)
    const int* offsets;       // [groups + 1]
    const int* shared;        // [groups]
    int groups, H;
    float c;                  // |scale| * log2(e), kSharedLeastFactor at least: the factor of the scores ...
    int negative;             // ... and whether the queries change sign
    // workspace
    float* prefix_parts;      // [2 * grid][kSharedColumns][D]
    f2* prefix_sums;
    float* tail_parts;        // [2 * wavefronts of the grid][heads_kept][D]
    f2* tail_sums;
    float* rows[2];           // [R][H][D] of prefix units, of tail units that one workgroup, or wavefront, did all of
    f2* row_sums[2];
    int4* requests;           // [R] (first request of the group, rows in common, group, length)
    int2* prefix_records;     // per unit: (first workgroup, or wavefront, last one); first -1: all of it is in `rows`
    int2* tail_records;
};

// Two probabilities as sums of two 16-bit numbers each: the first is cut off, the second what is left, rounded (bfloat16) or cut off (binary16).  Where the
// first is not zero the second is not either, since its product with an infinite value would be no number: bfloat16 takes what is left of a number larger by
// 2^-20, binary16 at least the smallest number there is, 2^-35 of the reference.  A binary16 probability below that is cut off, and both numbers are zero: were the second not,
// thousands of rows without weight would add up to what a row of small values that has all of it cannot stand beside.
template <bool BF16>
struct SharedPieces {
    static constexpr int kCount = 2;
    // A maximum is raised for scores by more than kSlack (in powers of two) above it; probabilities are scaled by 2^kShift: binary16 ones come up to 2^15 with the slack, bfloat16
    // ones up to 1, so that no value grows by its weight (values next to the largest number overflowed).
    static constexpr float kSlack = BF16 ? kRescaleSlack : 4.f, kShift = BF16 ? -kRescaleSlack : 11.f;
    static __device__ __forceinline__ unsigned first(float a, float b) {
        if constexpr (BF16) return __builtin_amdgcn_perm(__builtin_bit_cast(unsigned, b), __builtin_bit_cast(unsigned, a), 0x07060302u);
        else return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(a, b));
    }
    static __device__ __forceinline__ unsigned second(float a, float b, unsigned first) {
        if constexpr (BF16) {
            constexpr float kMore = 1.f + 0x1p-20f;
            return narrow<true>(__builtin_fmaf(a, kMore, -widen<true>(first, 0)), __builtin_fmaf(b, kMore, -widen<true>(first, 1)));
        } else {
            return __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_pkrtz(fmaxf(a - widen<false>(first, 0), fminf(a, 0x1p-24f)), fmaxf(b - widen<false>(first, 1), fminf(b, 0x1p-24f))));
        }
    }
};

// A column's new reference, of a raw score.  Scores below all numbers (of keys of the lowest value, as masks have them) leave a finite one: a difference from it is one, and their
// probabilities are 0.
__device__ __forceinline__ float shared_maximum(float raw, float factor) { return fmaxf(raw * factor, -0x1.fffffep127f); }
// Exponents are worked out in one step, raw score * factor + shift.  The product in it is not rounded, the one in the shift was, so that all rows' exponents are off by up to half of the reference's
// last bit.  That drops out of the quotient unless it is large: the best row's weight would be infinite, or 0.  Where a reference is beyond this number (last bit 2^-3), the scores are scaled and
// rounded first.
constexpr float kSharedFar = 0x1p20f;

// 32 rows in a wavefront's registers, as operands of both products.
template <int D>
struct RowsTile {
    u4 k[2][D / 32];             // of the first: row c of 16, which is key 4 (c % 4) + c / 4 of them, 32 elements each
    unsigned v[8][D / 32];       // of the second: rows 4 i + g, the lane's D / 16 elements c D / 16 .. of each
};

struct RowsPages {      // of the two halves of a tile
    int half[2];
    __device__ __forceinline__ RowsPages(const DecodeParams& p, const DecodeUnit& u, int tile) {
#pragma unroll
        for (int i = 0; i < 2; ++i) half[i] = u.pages[min(tile * 32 + i * 16, u.length - 1) >> p.shift];
    }
    __device__ __forceinline__ bool bad(const DecodeParams& p, int i) const { return (unsigned)half[i] >= (unsigned)p.pages; }
};

// A wavefront's part of a tail unit, or of a prefix unit of up to 32 columns: tiles of 32 rows in registers, the next one's loads behind the product that uses them up.  Tails alone, 64
// requests of up to 1000 rows and 256 of up to 2000: 22.4 and 87 us (read from the Infinity Cache in part); by workgroups, with tiles in LDS, 18.6 and 96; with a second set of registers 64 take 24.5.  V is read once and past the caches; K's rows come in four loads of 64
// bytes each, of which the caches join two (non-temporal: 10 % longer).
template <int D, bool BF16, int NB>
struct RowsState {
    using Pieces = SharedPieces<BF16>;
    int c, g;                // of the lane: lane % 16, lane / 16
    f4 o[NB][D / 16];        // lane (c, g): column c of block b, elements (4 g + i) * D / 16 + j in o[b][j][i]
    float l[NB];             // sums of the lane's own rows
    float limit[NB];         // raw score of the lane's column above which its reference has to be raised; -inf: there is none yet
    float shift[NB];         // kShift - reference: what scores times c are shifted by

    __device__ __forceinline__ RowsState(int lane) : c(lane & 15), g(lane >> 4) { clear(); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int b = 0; b < NB; ++b) {
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[b][j] = f4{0.f, 0.f, 0.f, 0.f};
            l[b] = 0.f;
            limit[b] = -INFINITY;
            shift[b] = 0.f;      // (any number will do: there is no score yet)
        }
    }
    __device__ __forceinline__ float reference(int b) const { return limit[b] == -INFINITY ? -INFINITY : -shift[b]; }

    __device__ __forceinline__ void load_k(const DecodeParams& p, const DecodeUnit& u, const RowsPages& pages, int tile, RowsTile<D>& to) const {
        const int mine = 4 * (c & 3) + (c >> 2);
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const char* const k = u.K + (pages.bad(p, half) ? 0 : pages.half[half]) * p.k_page + (long long)((tile * 32 + half * 16) & ((1 << p.shift) - 1)) * p.k_row;
#pragma unroll
            for (int x = 0; x < D / 32; ++x) to.k[half][x] = *reinterpret_cast<const u4*>(k + (mine * p.k_row + g * 16u) + x * 64);
        }
    }
    __device__ __forceinline__ void load_v(const DecodeParams& p, const DecodeUnit& u, const RowsPages& pages, int tile, RowsTile<D>& to) const {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const char* const v = u.V + (pages.bad(p, half) ? 0 : pages.half[half]) * p.v_page + (long long)((tile * 32 + half * 16) & ((1 << p.shift) - 1)) * p.v_row;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                typedef unsigned words __attribute__((ext_vector_type(D / 32)));
                const words w = __builtin_nontemporal_load(reinterpret_cast<const words*>(v + (long long)i * 4 * p.v_row + (g * p.v_row + c * (D / 8u))));
#pragma unroll
                for (int x = 0; x < D / 32; ++x) to.v[half * 4 + i][x] = w[x];
            }
        }
    }

    __device__ __forceinline__ void scores(const u4 (&q)[NB][D / 32], const RowsTile<D>& t, f4 (&s)[NB][2]) const {
#pragma unroll
        for (int x = 0; x < D / 32; ++x)
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half) s[b][half] = decode_mfma<BF16>(t.k[half][x], q[b][x], x ? s[b][half] : f4{0.f, 0.f, 0.f, 0.f});
    }

    // All columns see the rows u.low .. u.length - 1.  factor > 0.
    __device__ __forceinline__ void add(const DecodeParams& p, float factor, const DecodeUnit& u, const RowsPages& pages, int tile, f4 (&s)[NB][2], RowsTile<D>& t) {
        const int key0 = tile * 32;
        if (key0 < u.low || key0 + 32 > u.length || pages.bad(p, 0) || pages.bad(p, 1)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int key = key0 + 4 * i + g;
                const bool seen = key >= u.low && key < u.length;
#pragma unroll
                for (int b = 0; b < NB; ++b) s[b][i / 4][i % 4] = !seen ? -INFINITY : pages.bad(p, i / 4) ? __builtin_nanf("") : s[b][i / 4][i % 4];
                if (!seen) {      // whatever the row holds, it takes no part: 0 * NaN would
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) t.v[i][x] = 0;
                }
            }
        }
        float most[NB];
        bool above = false;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            // (maximumnum and not fmaxf: that would first make every score a quiet number)
            auto most3 = [](float x, float y, float z) { return __builtin_elementwise_maximumnum(__builtin_elementwise_maximumnum(x, y), z); };
            most[b] = __builtin_elementwise_maximumnum(most3(most3(most3(s[b][0][0], s[b][0][1], s[b][0][2]), s[b][0][3], s[b][1][0]), s[b][1][1], s[b][1][2]), s[b][1][3]);
            above = above || most[b] > limit[b];
        }
        if (__any(above)) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const float raw = head_max(most[b]);
                if (raw > limit[b]) {      // (all four lanes of a column alike)
                    const float M = shared_maximum(raw, factor), next = Pieces::kShift - M, fade = limit[b] == -INFINITY ? 1.f : fast_exp2(next - shift[b]);
                    limit[b] = score_limit(raw, M, factor, Pieces::kSlack);
                    shift[b] = next;
                    l[b] *= fade;
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) o[b][j] *= fade;
                }
            }
        }
        bool far = false;
#pragma unroll
        for (int b = 0; b < NB; ++b) far = far || fabsf(shift[b]) > kSharedFar;
        if (__any(far)) {
#pragma unroll
            for (int b = 0; b < NB; ++b)
#pragma unroll
                for (int half = 0; half < 2; ++half) s[b][half] *= factor;
            factor = 1.f;
        }
        u4 piece[NB][Pieces::kCount];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float x = fast_exp2(__builtin_fmaf(s[b][w / 2][w % 2 * 2], factor, shift[b])), y = fast_exp2(__builtin_fmaf(s[b][w / 2][w % 2 * 2 + 1], factor, shift[b]));
                l[b] += x + y;
                piece[b][0][w] = Pieces::first(x, y);
                piece[b][1][w] = Pieces::second(x, y, piece[b][0][w]);
            }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
            u4 a;      // element j of the lane's pieces of its eight rows
#pragma unroll
            for (int w = 0; w < 4; ++w) a[w] = __builtin_amdgcn_perm(t.v[2 * w + 1][j / 2], t.v[2 * w][j / 2], j % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
            for (int i = 0; i < Pieces::kCount; ++i)
#pragma unroll
                for (int b = 0; b < NB; ++b) o[b][j] = decode_mfma<BF16>(a, piece[b][i], o[b][j]);
        }
    }

    // Tiles first, first + stride, ... up to the one in front of `end`.
    __device__ __forceinline__ void add_tiles(const DecodeParams& p, float factor, const DecodeUnit& u, const u4 (&q)[NB][D / 32], int first, int stride, int end) {
        if (first >= end) return;
        RowsPages pages(p, u, first), ahead(p, u, first + stride);      // (behind the last one the last page again)
        RowsTile<D> rows;
        load_k(p, u, pages, first, rows);
        load_v(p, u, pages, first, rows);
        for (int tile = first;;) {
            const RowsPages further(p, u, tile + 2 * stride);
            const bool more = tile + stride < end;
            f4 s[NB][2];
            scores(q, rows, s);
            if (more) load_k(p, u, ahead, tile + stride, rows);
            add(p, factor, u, pages, tile, s, rows);
            if (!more) break;
            load_v(p, u, ahead, tile + stride, rows);
            pages = ahead;
            ahead = further;
            tile += stride;
        }
    }
};

// Units of more than 32 columns, up to 128: the workgroup takes tiles of 64 rows through LDS, K and V, two buffers each, and a wavefront has 32 columns of its own, so
// that there is nothing to join at the end (with up to 64 columns, CW = 2, two wavefronts share columns, each with every other 32 rows).  The operands of the
// second product come transposed from LDS (ds_read_b64_tr_b16, see NarrowMap for the places of the pieces of a row), in the order in which the
// first product leaves its rows: of 32 rows a lane holds 4 g + i and 16 + 4 g + i.
template <int D>
struct WideLane {
    static constexpr int kRowBytes = 2 * D, kPieces = D / 8, kRowsPerLoad = 64 / kPieces, kLoads = 16 / kRowsPerLoad;      // of a wavefront's 16 rows
    static constexpr int kTile = 64 * kRowBytes;      // of K or of V; a buffer holds K and then V
    int c, g;
    unsigned row, piece;             // the lane's row and piece of a load
    unsigned k_at[D / 32];           // in a tile of K: operands of the first 16 rows
    unsigned v_at[D / 16];           // in a tile of V
    __device__ __forceinline__ WideLane(int lane) {
        c = lane & 15;
        g = lane >> 4;
        row = lane / kPieces;
        piece = (lane % kPieces ^ NarrowMap<D>::swz(row)) * 16;
        const int e = c >> 2, chunk = c & 3;      // transposed: row and 8 bytes of it that the lane names
#pragma unroll
        for (int x = 0; x < D / 32; ++x) k_at[x] = c * kRowBytes + (((4 * x + g) ^ NarrowMap<D>::swz(c)) * 16);
#pragma unroll
        for (int j = 0; j < D / 16; ++j) v_at[j] = (4 * g + e) * kRowBytes + (((2 * j + (chunk >> 1)) ^ NarrowMap<D>::swz(4 * g + e)) * 16) + 8 * (chunk & 1);
    }
};

struct WidePages {      // of a tile's rows, 16 at a time
    int part[4], mine;      // mine: of those that the wavefront fetches
    __device__ __forceinline__ WidePages(const DecodeParams& p, const DecodeUnit& u, int tile, int wave) {
        auto of = [&](int i) { return u.pages[min(tile * 64 + i * 16, u.length - 1) >> p.shift]; };
#pragma unroll
        for (int i = 0; i < 4; ++i) part[i] = of(i);
        mine = of(wave);
    }
};

template <int D, bool BF16, int CW>
struct WideState {
    using L = WideLane<D>;
    using Pieces = SharedPieces<BF16>;
    static constexpr int SUBS = CW == 4 ? 2 : 1;      // 32 rows of a tile at a time
    f4 o[2][D / 16];         // lane (c, g): column c of block b, elements 16 j + 4 g + i in o[b][j][i]
    float l[2], limit[2], shift[2];      // as in RowsState

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[b][j] = f4{0.f, 0.f, 0.f, 0.f};
            l[b] = 0.f;
            limit[b] = -INFINITY;
            shift[b] = 0.f;      // (any number will do: there is no score yet)
        }
    }
    __device__ __forceinline__ float reference(int b) const { return limit[b] == -INFINITY ? -INFINITY : -shift[b]; }

    // The wavefront's 16 rows of a tile on their way to LDS; rows behind the last one become zeros, 0 * NaN would be none.
    static __device__ __forceinline__ void fetch(const DecodeParams& p, const L& lane, const DecodeUnit& u, const WidePages& pages, int tile, int wave, LDS_PTR(char) buffer) {
        const int row0 = tile * 64 + wave * 16;
        LDS_PTR(char) const to = buffer + wave * 16 * L::kRowBytes;
        if (row0 >= u.length) {
#pragma unroll
            for (int i = 0; i < L::kLoads; ++i)
                *(LDS_PTR(u4))(to + L::kTile + i * 1024 + lane_now() * 16) = u4{0, 0, 0, 0};
            return;
        }
        const int page = __builtin_amdgcn_readfirstlane((unsigned)pages.mine >= (unsigned)p.pages ? 0 : pages.mine);
        const int row = row0 & ((1 << p.shift) - 1);
        const char* const k = u.K + page * p.k_page + (long long)row * p.k_row;
        const char* const v = u.V + page * p.v_page + (long long)row * p.v_row;
#pragma unroll
        for (int i = 0; i < L::kLoads; ++i)
            load_to_lds_16B(k + (long long)i * L::kRowsPerLoad * p.k_row, lane.row * p.k_row + (lane.piece ^ NarrowMap<D>::swz(i * L::kRowsPerLoad) * 16),
                            (unsigned)(uintptr_t)to + i * 1024);
#pragma unroll
        for (int i = 0; i < L::kLoads; ++i)
            load_to_lds_16B(v + (long long)i * L::kRowsPerLoad * p.v_row, lane.row * p.v_row + (lane.piece ^ NarrowMap<D>::swz(i * L::kRowsPerLoad) * 16),
                            (unsigned)(uintptr_t)to + L::kTile + i * 1024);
    }

    // Takes in a tile that is in LDS.  sub0: the 32 rows of it that a wavefront begins with.
    __device__ __forceinline__ void add(const DecodeParams& p, float c, const L& lane, const DecodeUnit& u, const u4 (&q)[2][D / 32], const WidePages& pages, int tile,
                                        int sub0, LDS_PTR(char) buffer) {
        LDS_PTR(char) const kv = buffer + sub0 * 32 * L::kRowBytes;
        f4 s[SUBS][2][2];
        // K's operands are read some ahead of the MFMAs (left to the compiler each is waited for: 256 requests, 32768 rows in common 221 -> 207 us)
        constexpr int kOperands = SUBS * (D / 16), kAhead = 4;      // of (32 rows, 16 of them, 32 elements)
        __builtin_amdgcn_s_setprio(2);      // (between here and the next one wait those that share the SIMD and have no MFMAs to issue)
        u4 k[kOperands];
        auto k_operand = [&](int n) {
            const int sub = n / (D / 16), half = n % 2, x = n / 2 % (D / 32);
            k[n] = *(LDS_PTR(const u4))(kv + lane.k_at[x] + (sub * 32 + half * 16) * L::kRowBytes);
        };
#pragma unroll
        for (int n = 0; n < kAhead; ++n) k_operand(n);
#pragma unroll
        for (int n = 0; n < kOperands; ++n) {
            const int sub = n / (D / 16), half = n % 2, x = n / 2 % (D / 32);
            if (n + kAhead < kOperands) k_operand(n + kAhead);
#pragma unroll
            for (int b = 0; b < 2; ++b) s[sub][b][half] = decode_mfma<BF16>(k[n], q[b][x], x ? s[sub][b][half] : f4{0.f, 0.f, 0.f, 0.f});
            __builtin_amdgcn_sched_barrier(0);
        }
        u4 a[D / 16];
        auto v_operand = [&](int sub, int j) {
            LDS_PTR(char) const at = kv + L::kTile + lane.v_at[j] + sub * 32 * L::kRowBytes;
            const u2 low = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s4))at));
            const u2 high = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_PTR(s4))(at + 16 * L::kRowBytes)));
            a[j] = u4{low[0], low[1], high[0], high[1]};
        };
#pragma unroll
        for (int j = 0; j < D / 16; ++j) v_operand(0, j);
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) bad = bad || (unsigned)pages.part[i] >= (unsigned)p.pages;
        if (bad || (tile + 1) * 64 > u.length) {
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
                for (int half = 0; half < 2; ++half) {      // 16 rows: all there or none, all of one page
                    const int part = 2 * (sub0 + sub) + half;
                    const int low = pages.part[2 * sub + half], high = pages.part[2 + half], page = SUBS == 2 || sub0 == 0 ? low : high;
                    const bool seen = tile * 64 + part * 16 < u.length;
                    if (seen && (unsigned)page < (unsigned)p.pages) continue;
                    const float none = seen ? __builtin_nanf("") : -INFINITY;
#pragma unroll
                    for (int b = 0; b < 2; ++b) s[sub][b][half] = f4{none, none, none, none};
                }
        }
        float most[2];
        bool above = false;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            // (maximumnum and not fmaxf: that would first make every score a quiet number)
            auto most3 = [](float x, float y, float z) { return __builtin_elementwise_maximumnum(__builtin_elementwise_maximumnum(x, y), z); };
            most[b] = -INFINITY;
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
                for (int half = 0; half < 2; ++half) most[b] = most3(most3(most[b], s[sub][b][half][0], s[sub][b][half][1]), s[sub][b][half][2], s[sub][b][half][3]);
            above = above || most[b] > limit[b];
        }
        if (__any(above)) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const float t = head_max(most[b]);
                if (t > limit[b]) {      // (all four lanes of a column alike)
                    const float M = shared_maximum(t, c), next = Pieces::kShift - M, fade = limit[b] == -INFINITY ? 1.f : fast_exp2(next - shift[b]);
                    limit[b] = score_limit(t, M, c, Pieces::kSlack);
                    shift[b] = next;
                    l[b] *= fade;
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) o[b][j] *= fade;
                }
            }
        }
        if (__any(fabsf(shift[0]) > kSharedFar || fabsf(shift[1]) > kSharedFar)) {
#pragma unroll
            for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int half = 0; half < 2; ++half) s[sub][b][half] *= c;
            c = 1.f;
        }
        __builtin_amdgcn_s_setprio(0);
        u4 piece[SUBS][2][Pieces::kCount];
        float x[2];
        auto softmax = [&](int sub, int step) {      // 32 steps: of each pair of rows the exponents, the powers, their two parts
            const int b = step / 16, w = step / 4 % 4, at = w % 2 * 2;
            if (step % 4 == 0) {
#pragma unroll
                for (int i = 0; i < 2; ++i) x[i] = __builtin_fmaf(s[sub][b][w / 2][at + i], c, shift[b]);
            } else if (step % 4 == 1) {
#pragma unroll
                for (int i = 0; i < 2; ++i) x[i] = fast_exp2(x[i]);
            } else if (step % 4 == 2) {
                l[b] += x[0] + x[1];
                piece[sub][b][0][w] = Pieces::first(x[0], x[1]);
            } else {
                piece[sub][b][1][w] = Pieces::second(x[0], x[1], piece[sub][b][0][w]);
            }
        };
#pragma unroll
        for (int step = 0; step < 32; ++step) softmax(0, step);
        __builtin_amdgcn_s_setprio(2);
#pragma unroll
        for (int sub = 0; sub < SUBS; ++sub)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
#pragma unroll
                for (int n = 0; n < 4; ++n) {      // the second 32 rows' exponentials stand between the MFMAs of the first ones
                    o[n % 2][j] = decode_mfma<BF16>(a[j], piece[sub][n % 2][n / 2], o[n % 2][j]);
                    if (sub + 1 < SUBS) {
                        constexpr int kSteps = 32 * 16 / D;      // to an operand
#pragma unroll
                        for (int step = j * kSteps + n * kSteps / 4; step < j * kSteps + (n + 1) * kSteps / 4; ++step) softmax(sub + 1, step);
                    }
                }
                if (sub + 1 < SUBS) {
                    v_operand(sub + 1, j);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
    }
};

// The wavefronts' parts of up to 16 columns, added up; store(column, element / 4, m, l, o) gets the sums.
template <int D, typename STORE>
__device__ __forceinline__ void join_waves(char (*area)[kDecodeHeads * (D + 4) * 4], float (*m_of)[kDecodeHeads], float (*l_of)[kDecodeHeads], const f4 (&state)[D / 16],
                                           float state_m, float sum, int wave, int columns, STORE&& store) {
    constexpr int kPitch = D + 4;
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
    all = __builtin_amdgcn_readfirstlane(all);
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

template <int D, bool BF16>
__global__ __launch_bounds__(kSharedThreads, 2) void decode_shared_kernel(SharedParams p) {
    constexpr int kPitch = D + 4, kArea = kDecodeHeads * kPitch * 4, kColumns = kSharedColumns, kBuffer = 2 * WideLane<D>::kTile;
    static_assert(kColumns == 32 * kDecodeWaves, "a wavefront has 32 columns");
    __shared__ __align__(16) char memory[std::max(kDecodeWaves * kArea, 2 * kBuffer)];
    auto& area = *reinterpret_cast<char (*)[kDecodeWaves][kArea]>(memory);      // a wavefront's own
    __shared__ float m_of[kDecodeWaves][kDecodeHeads], l_of[kDecodeWaves][kDecodeHeads];
    __shared__ int of_wave[2][kDecodeWaves];
    __shared__ SharedStart start_prefix, start_tail[kDecodeWaves];
    __shared__ int falls;
    extern __shared__ int lists[];      // offsets [groups + 1], rows in common [groups], first request that is not empty [groups], lengths [R]
    const DecodeParams& d = p.d;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), block = blockIdx.x, grid = gridDim.x;
    const SharedGroups in = {lists, lists + p.groups + 1, lists + 2 * p.groups + 1, p.groups};
    int* const lengths = lists + 3 * p.groups + 1;

    // ---- the groups (the first numbers of all lists on their way at once)
    const int offset0 = tid <= p.groups ? p.offsets[tid] : 0, shared0 = tid < p.groups ? p.shared[tid] : 0, length0 = tid < d.R ? d.lengths[tid] : 0;
    if (tid == 0) falls = 0;
    for (int g = tid; g <= p.groups; g += kSharedThreads) in.offsets[g] = min(max(g == tid ? offset0 : p.offsets[g], 0), d.R);
    for (int g = tid; g < p.groups; g += kSharedThreads) {
        in.common[g] = g == tid ? shared0 : p.shared[g];
        in.lead[g] = d.R;
    }
    for (int r = tid; r < d.R; r += kSharedThreads) lengths[r] = min(max(r == tid ? length0 : d.lengths[r], 0), d.capacity);
    __syncthreads();
    for (int g = tid; g < p.groups; g += kSharedThreads)
        if (in.offsets[g] > in.offsets[g + 1]) falls = 1;
    for (int r = tid; r < d.R; r += kSharedThreads) {
        const int g = in.of_request(r);
        if (lengths[r] && g >= 0) {
            atomicMin(&in.common[g], lengths[r]);
            atomicMin(&in.lead[g], r);
        }
    }
    __syncthreads();
    auto blocks_of = [&](int g) { return ((in.offsets[g + 1] - in.offsets[g]) * d.group + kColumns - 1) / kColumns; };
    auto prefix_steps = [&](int g) { return (in.common[g] + kDecodeStep - 1) / kDecodeStep; };
    const int each_group = (p.groups + kSharedThreads - 1) / kSharedThreads, g0 = tid * each_group;
    int mine_prefix = 0;
    for (int i = 0; i < each_group; ++i) {
        const int g = g0 + i;
        if (g >= p.groups) break;
        const int size = in.offsets[g + 1] - in.offsets[g], common = in.lead[g] < d.R && size > 1 && !falls ? max(in.common[g], 0) >> d.shift << d.shift : 0;
        in.common[g] = common;
        if (common) mine_prefix += prefix_steps(g) * blocks_of(g) * d.units;
    }
    int total_prefix, total_tail;
    int before_prefix = shared_before(mine_prefix, of_wave[0], total_prefix);      // (a barrier in it: what the groups have in common is there)
    // ---- the requests
    auto tail_from = [&](int g) { return g >= 0 ? in.common[g] : 0; };
    auto tail_tiles = [&](int length, int from) { return length > from ? (length - 1) / 32 - from / 32 + 1 : 0; };
    const int each = (d.R + kSharedThreads - 1) / kSharedThreads, r0 = tid * each;
    const int units = d.units * d.head_groups;
    int mine_tail = 0;
    for (int i = 0; i < each; ++i) {
        const int r = r0 + i;
        if (r >= d.R) break;
        const int g = in.of_request(r), from = tail_from(g);
        mine_tail += tail_tiles(lengths[r], from) * units;
        if (block == 0) p.requests[r] = int4{g >= 0 ? in.offsets[g] : r, from, max(g, 0), lengths[r]};
    }
    int before_tail = shared_before(mine_tail, of_wave[1], total_tail);
    // ---- who does what.  Every workgroup takes its share of both kinds, or each does one of them: what ends sooner by an estimate that counts a step of a prefix as kStep and a
    // tile of a tail as kTile half microseconds (groups of the mean size have wide units or not; with 7 or 14 for 10, or 3 or 6 for kTile,
    // 64 requests behind 8192 rows take 42 instead of 41 us and the join 9 instead of 8).  (With much to do it is the first, where the matrix cores and the memory have work at the same time.)
    const int kStep = d.R * d.group > 32 * p.groups ? 10 : 4;
    constexpr int kTile = 4, kMuch = 8;
    auto parts = [](int all, int takers) { return (int)(((unsigned)all + (unsigned)takers - 1) / (unsigned)takers); };
    int prefix_takers = grid, tail_takers = grid;
    const bool much = total_prefix >= kMuch * grid;
    if (!much && total_prefix && total_tail) {
        const float prefix_cost = (float)total_prefix * kStep, part = prefix_cost / (prefix_cost + (float)total_tail * (kTile / (float)kDecodeWaves));
        const int steps = parts(total_prefix, min(max((int)(part * (float)grid), 1), grid - 1)), takers = parts(total_prefix, steps);
        if (max(steps * kStep, parts(total_tail, kDecodeWaves * (grid - takers)) * kTile) < parts(total_prefix, grid) * kStep + parts(total_tail, kDecodeWaves * grid) * kTile) {
            prefix_takers = takers;
            tail_takers = grid - takers;
        }
    }
    const int waves = tail_takers * kDecodeWaves;      // that take tails
    const int share_prefix = parts(total_prefix, prefix_takers), share_tail = parts(total_tail, waves);
    // Workgroups go round the XCDs; where they have much to do, those of one XCD take neighbouring shares, which read the same rows where a group has several units.
    const int wp = much ? block % 8 * (grid / 8) + block / 8 : block;
    const int at_prefix = wp < prefix_takers ? wp * share_prefix : total_prefix;      // (below the total and twice the grid, like those of the tails)
    int left_prefix = min(share_prefix, total_prefix - at_prefix);
    if (left_prefix > 0 && at_prefix >= before_prefix && at_prefix < before_prefix + mine_prefix) {
        int g = g0;
        for (;; ++g) {
            const int steps = in.common[g] ? prefix_steps(g) * blocks_of(g) * d.units : 0;
            if (at_prefix < before_prefix + steps) break;
            before_prefix += steps;
        }
        start_prefix = SharedStart{g, at_prefix - before_prefix};
    }
    const int wt = (grid - 1 - block) * kDecodeWaves;      // the first wavefront's number among those that take tails
    for (int w = 0; w < kDecodeWaves; ++w) {
        if (wt >= waves) break;
        const int at = (wt + w) * share_tail;
        if (at < before_tail || at >= before_tail + mine_tail) continue;
        int r = r0, before = before_tail;
        for (;; ++r) {
            const int tiles = tail_tiles(lengths[r], tail_from(in.of_request(r))) * units;
            if (at < before + tiles) break;
            before += tiles;
        }
        start_tail[w] = SharedStart{r, at - before};
    }
    __syncthreads();

    auto prefixes = [&]() {
        if (left_prefix <= 0) return;
        int g = __builtin_amdgcn_readfirstlane(start_prefix.item);
        const int inside = __builtin_amdgcn_readfirstlane(start_prefix.inside);
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
            const int now = tid & 63, c = now & 15, g4 = now >> 4;
            auto query = [&](u4 (&q)[D / 32], int column) {      // the operands of a lane's column
#pragma unroll
                for (int x = 0; x < D / 32; ++x) q[x] = u4{0, 0, 0, 0};
                if (column < columns) {
                    int r;
                    const int head = row_of(column, r);
                    const char* const from = d.Q + r * d.q_request + head * d.q_head + g4 * 16;
#pragma unroll
                    for (int x = 0; x < D / 32; ++x) q[x] = *reinterpret_cast<const u4*>(from + x * 64) ^ (p.negative ? 0x80008000u : 0u);
                }
            };
            const int length = __builtin_amdgcn_readfirstlane(in.common[g]), lead = __builtin_amdgcn_readfirstlane(in.lead[g]);
            const DecodeUnit u = {d.K + unit * d.k_head, d.V + unit * d.v_head,
                                  (const __attribute__((address_space(4))) int*)(uintptr_t)(d.table + lead * d.table_stride), 0, length};
            const bool whole = t0 == 0 && t1 == steps;
            const long long place = 2 * wp + (t0 == 0 ? 1 : 0);
            // Where the sums of a column go: to the unit's rows, or to the workgroup's place for parts.
            auto destination = [&](int column, float*& to, f2*& sums) {
                long long row = place * kColumns + column;
                to = p.prefix_parts;
                sums = p.prefix_sums;
                if (whole) {
                    int r;
                    const int head = row_of(column, r);
                    row = (long long)r * p.H + head;
                    to = p.rows[0];
                    sums = p.row_sums[0];
                }
                to += row * D;
                sums += row;
            };
            auto wide_part = [&](auto width) {
                constexpr int CW = decltype(width)::value;
                const WideLane<D> at(now);
                const int column0 = wave % CW * 32, sub0 = wave / CW, tiles = min(2 * t1, (length + 63) / 64);
                u4 q[2][D / 32];
#pragma unroll
                for (int b = 0; b < 2; ++b) query(q[b], column0 + 16 * b + c);
                WideState<D, BF16, CW> state;
                state.clear();
                LDS_PTR(char) const buffers = (LDS_PTR(char))memory;
                __syncthreads();      // (others may still read what was there)
                int tile = 2 * t0;
                WidePages pages(d, u, tile, wave), ahead(d, u, tile + 1, wave);      // (behind the last one the last page again)
                state.fetch(d, at, u, pages, tile, wave, buffers);
                for (; tile < tiles; ++tile) {
                    landed_barrier<0>();
                    if (tile + 1 < tiles) state.fetch(d, at, u, ahead, tile + 1, wave, buffers + ((tile + 1) & 1) * kBuffer);
                    const WidePages further(d, u, tile + 2, wave);
                    state.add(d, p.c, at, u, q, pages, tile, sub0, buffers + (tile & 1) * kBuffer);
                    pages = ahead;
                    ahead = further;
                }
                __builtin_amdgcn_s_setprio(0);
                float l[2], m[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    l[b] = head_sum(state.l[b]);
                    m[b] = state.reference(b);
                }
                if constexpr (CW == 2) {      // the other 32 rows of each tile
                    float* const other = reinterpret_cast<float*>(memory) + wave % 2 * 32 * kPitch;
                    float* const sums = reinterpret_cast<float*>(memory) + 2 * 32 * kPitch + wave % 2 * 64;
                    __syncthreads();
                    if (sub0 == 1) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
#pragma unroll
                            for (int j = 0; j < D / 16; ++j) *reinterpret_cast<f4*>(other + (16 * b + c) * kPitch + 16 * j + 4 * g4) = state.o[b][j];
                            if (g4 == 0) {
                                sums[16 * b + c] = m[b];
                                sums[32 + 16 * b + c] = l[b];
                            }
                        }
                    }
                    __syncthreads();
                    if (sub0 == 1) return;
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const float m1 = sums[16 * b + c], most = fmaxf(m[b], m1), reference = most == -INFINITY ? 0.f : most;
                        const float f = fast_exp2(m[b] - reference), f1 = fast_exp2(m1 - reference);
                        m[b] = most;
                        l[b] = f * l[b] + f1 * sums[32 + 16 * b + c];
#pragma unroll
                        for (int j = 0; j < D / 16; ++j) state.o[b][j] = f * state.o[b][j] + f1 * *reinterpret_cast<const f4*>(other + (16 * b + c) * kPitch + 16 * j + 4 * g4);
                    }
                }
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int column = column0 + 16 * b + c;
                    if (column >= columns) continue;
                    float* to;
                    f2* sums;
                    destination(column, to, sums);
#pragma unroll
                    for (int j = 0; j < D / 16; ++j) *reinterpret_cast<f4*>(to + 16 * j + 4 * g4) = state.o[b][j];
                    if (g4 == 0) *sums = f2{m[b], l[b]};
                }
            };
            auto narrow_part = [&](auto width) {
                constexpr int BLOCKS = decltype(width)::value;
                __syncthreads();      // (others may still read tiles of a wide unit)
                u4 q[BLOCKS][D / 32];
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) query(q[b], 16 * b + c);
                RowsState<D, BF16, BLOCKS> state(now);
                state.add_tiles(d, p.c, u, q, t0 * kDecodeWaves + wave, kDecodeWaves, min(t1 * kDecodeWaves, (length + 31) / 32));
#pragma unroll
                for (int b = 0; b < BLOCKS; ++b) {
                    if (16 * b >= columns) continue;
                    join_waves<D>(area, m_of, l_of, state.o[b], state.reference(b), head_sum(state.l[b]), wave, min(16, columns - 16 * b), [&](int column, int at4, float m, float l, f4 o) {
                        float* to;
                        f2* sums;
                        destination(16 * b + column, to, sums);
                        *reinterpret_cast<f4*>(to + at4) = o;
                        if (at4 == 0) *sums = f2{m, l};
                    });
                }
            };
            // a unit computes no more columns than it has, up to 16, 32, 64
            if (columns > 64) wide_part(std::integral_constant<int, 4>{});
            else if (columns > 32) wide_part(std::integral_constant<int, 2>{});
            else if (columns > 16) narrow_part(std::integral_constant<int, 2>{});
            else narrow_part(std::integral_constant<int, 1>{});
            if (t0 == 0 && tid == 0) {
                const long long record = ((long long)begin * d.group / kColumns + g + (part - unit * blocks)) * d.units + unit;
                p.prefix_records[record] = whole ? int2{-1, 0} : int2{wp, min(wp + (steps - t1 + share_prefix - 1) / share_prefix, prefix_takers - 1)};
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
    auto tails = [&]() {      // every wavefront by itself, tile by tile, whatever units they are of: the next one's rows and queries are on their way meanwhile
        const int place0 = wt + wave;
        int left = place0 < waves ? min(share_tail, total_tail - place0 * share_tail) : 0;
        if (left <= 0) return;
        const int now = tid & 63, c = now & 15, g4 = now >> 4;
        struct Item {      // a tile of a unit
            int r, part, tile, end, from, length;      // part: unit * head groups + head group; end: of the unit's tiles
            bool first;                                // of the unit
        };
        auto request = [&](Item& to, int r) {
            to.r = r;
            to.length = __builtin_amdgcn_readfirstlane(lengths[r]);
            to.from = __builtin_amdgcn_readfirstlane(tail_from(in.of_request(r)));
            to.end = (to.length + 31) / 32;
            return tail_tiles(to.length, to.from);
        };
        auto behind = [&](const Item& x) {      // the next one; behind the last one of all it again
            Item y = x;
            y.first = false;
            if (++y.tile < y.end) return y;
            y.first = true;
            if (++y.part == units) {
                y.part = 0;
                do {
                    if (y.r + 1 >= d.R) return x;
                } while (request(y, y.r + 1) == 0);
            }
            y.tile = y.from / 32;
            return y;
        };
        auto unit_of = [&](const Item& x) {
            const int unit = (unsigned)x.part / (unsigned)d.head_groups;
            return DecodeUnit{d.K + unit * d.k_head, d.V + unit * d.v_head,
                              (const __attribute__((address_space(4))) int*)(uintptr_t)(d.table + x.r * d.table_stride), x.from, x.length};
        };
        auto heads_of = [&](const Item& x, int& head0) {
            const int unit = (unsigned)x.part / (unsigned)d.head_groups, group0 = (x.part - unit * d.head_groups) * kDecodeHeads;
            head0 = unit * d.group + group0;
            return min(kDecodeHeads, d.group - group0);
        };
        auto queries = [&](u4 (&q)[1][D / 32], const Item& x) {
            int head0;
            const bool mine = c < heads_of(x, head0);
            const char* const row = d.Q + x.r * d.q_request + (long long)(head0 + (mine ? c : 0)) * d.q_head + g4 * 16;
#pragma unroll
            for (int i = 0; i < D / 32; ++i) {
                q[0][i] = *reinterpret_cast<const u4*>(row + i * 64) ^ (p.negative ? 0x80008000u : 0u);
                if (!mine) q[0][i] = u4{0, 0, 0, 0};
            }
        };
        Item item;
        const int tiles = request(item, __builtin_amdgcn_readfirstlane(start_tail[wave].item)), inside = __builtin_amdgcn_readfirstlane(start_tail[wave].inside);
        item.part = (unsigned)inside / (unsigned)tiles;
        item.tile = item.from / 32 + inside - item.part * tiles;
        item.first = item.tile == item.from / 32;
        bool begun_here = item.first;
        Item next = behind(item);
        RowsState<D, BF16, 1> state(now);
        RowsTile<D> rows;
        u4 q[1][D / 32];
        DecodeUnit u = unit_of(item);
        RowsPages pages(d, u, item.tile), ahead(d, unit_of(next), next.tile);
        queries(q, item);
        state.load_k(d, u, pages, item.tile, rows);
        state.load_v(d, u, pages, item.tile, rows);
        for (;;) {
            const Item further = behind(next);
            const DecodeUnit u_next = unit_of(next);
            const RowsPages pages_further(d, unit_of(further), further.tile);
            const bool more = --left > 0, ends = !more || next.first;
            f4 s[1][2];
            state.scores(q, rows, s);
            if (more) {
                state.load_k(d, u_next, ahead, next.tile, rows);
                if (next.first) queries(q, next);
            }
            state.add(d, p.c, u, pages, item.tile, s, rows);
            if (more) state.load_v(d, u_next, ahead, next.tile, rows);
            if (ends) {
                const bool whole = begun_here && item.tile + 1 == item.end;
                const float l = head_sum(state.l[0]);
                int head0;
                const int heads = heads_of(item, head0);
                if (c < heads) {
                    const long long row = whole ? (long long)item.r * p.H + head0 + c : (2LL * place0 + (begun_here ? 1 : 0)) * d.heads_kept + c;
                    float* const to = (whole ? p.rows[1] : p.tail_parts) + row * D;
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int j = 0; j < D / 16; j += 4)
                            *reinterpret_cast<f4*>(to + (4 * g4 + i) * (D / 16) + j) = f4{state.o[0][j][i], state.o[0][j + 1][i], state.o[0][j + 2][i], state.o[0][j + 3][i]};
                    if (g4 == 0) (whole ? p.row_sums[1] : p.tail_sums)[row] = f2{state.reference(0), l};
                }
                if (begun_here && now == 0)
                    p.tail_records[(long long)item.r * units + item.part] = whole ? int2{-1, 0} : int2{place0, min(place0 + parts(item.end - item.tile - 1, share_tail), waves - 1)};
                state.clear();
                begun_here = true;
            }
            if (!more) break;
            item = next;
            next = further;
            u = u_next;
            pages = ahead;
            ahead = pages_further;
        }
    };
    // (blocks go round the XCDs and, in them, round the 32 compute units)
    const bool tails_first = block / 256 % 2 != 0;
    for (int i = 0; i < 2; ++i) {
        if (tails_first == (i != 0)) prefixes();
        else tails();
    }
}

// Joins for every row of O the parts of its prefix unit and of its tail unit.  A row is D / 4 threads'; GROUPS of them go over every GROUPS-th part.
constexpr int kSharedJoinThreads = 256, kSharedJoinAhead = 4;

template <int D, int GROUPS>
__global__ __launch_bounds__(kSharedJoinThreads) void decode_shared_join_kernel(SharedParams p, int grid) {
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
    auto add = [&](int2 record, const float* parts, const f2* sums, int kept, int column, const float* rows, const f2* row_sums, int takers) {
        const bool whole = record.x < 0;
        const int first = whole ? 0 : max(record.x, 0), last = whole ? 0 : min(record.y, takers - 1);
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
    const int at = (r - request.x) * d.group + in_unit, block = at / kSharedColumns, head_group = in_unit / kDecodeHeads;
    int2 prefix = {0, -1}, tail = {0, -1};
    if (common) prefix = p.prefix_records[((long long)request.x * d.group / kSharedColumns + request.z + block) * d.units + unit];
    if (behind) tail = p.tail_records[((long long)r * d.units + unit) * d.head_groups + head_group];
    if (common) add(prefix, p.prefix_parts, p.prefix_sums, kSharedColumns, at - block * kSharedColumns, p.rows[0], p.row_sums[0], grid);
    if (behind) add(tail, p.tail_parts, p.tail_sums, d.heads_kept, in_unit - head_group * kDecodeHeads, p.rows[1], p.row_sums[1], grid * kDecodeWaves);
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

// The workspace, in bytes from the front.
struct SharedWorkspace {
    size_t prefix_sums, tail_parts, tail_sums, rows[2], row_sums[2], requests, prefix_records, tail_records, all;
    SharedWorkspace(const DecodePlan& plan, int R, int H, int groups, int d) {
        const size_t places = 2 * kSharedGrid, n = (size_t)R * H;
        size_t at = places * kSharedColumns * d * 4;
        auto next = [&](size_t& where, size_t bytes) { where = at; at += (bytes + 15) / 16 * 16; };
        next(prefix_sums, places * kSharedColumns * 8);
        next(tail_parts, kDecodeWaves * places * plan.heads_kept * d * 4);
        next(tail_sums, kDecodeWaves * places * plan.heads_kept * 8);
        for (int i = 0; i < 2; ++i) next(rows[i], n * d * 4);
        for (int i = 0; i < 2; ++i) next(row_sums[i], n * 8);
        next(requests, 16 * (size_t)R);
        next(prefix_records, 8 * ((size_t)R * plan.group / kSharedColumns + groups + 1) * plan.units);
        next(tail_records, 8 * (size_t)R * plan.units * plan.head_groups);
        all = at;
    }
};

int shared_plan(const sawattn_kv_cache* cache, int R, int H, int groups, int max_pages, DecodePlan* plan) {
    const int rc = decode_plan(cache, R, H, max_pages, 0, plan);
    if (rc != SAWATTN_OK) return rc;
    if (groups <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "groups must be positive");
    if (R > SAWATTN_MOST_REQUESTS || groups > SAWATTN_MOST_REQUESTS) return fail(SAWATTN_ERR_UNSUPPORTED, "more requests or groups than SAWATTN_MOST_REQUESTS");
    const double tiles = std::ceil((double)max_pages * cache->page_size / 32);
    if (tiles * R * H >= 2147483648.0 - 4.0 * kDecodeWaves * kSharedGrid) return fail(SAWATTN_ERR_INVALID_ARG, "R*H*ceil(max_pages*page_size/32) must be below 2^31 - 8192");
    return SAWATTN_OK;
}

template <int D, bool BF16>
int launch_shared(const SharedParams& p, int grid, hipStream_t stream) {
    hipLaunchKernelGGL((decode_shared_kernel<D, BF16>), dim3(grid), dim3(kSharedThreads), sizeof(int) * (3 * (size_t)p.groups + 1 + p.d.R), stream, p);
    const int rc = launched("attn_decode_shared");
    if (rc != SAWATTN_OK) return rc;
    const int rows = p.d.R * p.H;
    constexpr int kAcross = D / 4, kRows4 = kSharedJoinThreads / (4 * kAcross), kRows1 = kSharedJoinThreads / kAcross;
    // (2080 rows of 5 parts 7.9 us with 4, 8.7 with 1; 8192 of 4 17 and 11)
    if (rows <= 4096) hipLaunchKernelGGL((decode_shared_join_kernel<D, 4>), dim3((rows + kRows4 - 1) / kRows4), dim3(kSharedJoinThreads), 0, stream, p, grid);
    else hipLaunchKernelGGL((decode_shared_join_kernel<D, 1>), dim3((rows + kRows1 - 1) / kRows1), dim3(kSharedJoinThreads), 0, stream, p, grid);
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
    size_t alone = 0;
    rc = attn_decode_workspace_bytes(cache, R, H, max_pages, &alone);
    if (rc != SAWATTN_OK) return rc;
    *bytes = std::max(SharedWorkspace(plan, R, H, groups, cache->d).all, alone);
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
    size_t need = 0;
    rc = attn_decode_shared_workspace_bytes(cache, R, H, groups, max_pages, &need);
    if (rc != SAWATTN_OK) return rc;
    if (!Q || !O || !table || !lengths || !group_offsets || !shared || !workspace)
        return fail(SAWATTN_ERR_INVALID_ARG, "Q, O, table, lengths, group_offsets, shared and workspace must be non-null");
    if (((uintptr_t)group_offsets | (uintptr_t)shared) & 3u) return fail(SAWATTN_ERR_INVALID_ARG, "group_offsets and shared must be 4-byte aligned");
    if (workspace_bytes < need) return fail(SAWATTN_ERR_INVALID_ARG, "workspace is smaller than attn_decode_shared_workspace_bytes reports");
    SharedParams p{};
    rc = decode_params(Q, q_request, q_head, O, o_request, o_head, o_dtype, cache, table, table_stride, max_pages, lengths, R, H, scale, 0, workspace, workspace_bytes, need,
                       plan, &p.d);
    if (rc != SAWATTN_OK) return rc;
    auto extent = [](int n, int64_t stride) { return n > 1 ? (unsigned long long)(n - 1) * stride : 0ull; };
    const Range o(O, (o_dtype == SAWATTN_F32 ? 4 : 2) * (extent(R, o_request) + extent(H, o_head) + d)), scratch(workspace, need);
    for (const Range& i : {Range(group_offsets, 4ull * (groups + 1)), Range(shared, 4ull * groups)})
        if (o.meets(i) || scratch.meets(i)) return fail(SAWATTN_ERR_INVALID_ARG, "O and workspace must not overlap what is read");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if ((double)R * plan.units * p.d.capacity * 4 * d <= (double)(plan.direct ? kSharedFewDirect : kSharedFew) || std::fabs(p.d.c) < kSharedLeastFactor)
        return run_decode(p.d, plan, H, d, cache->dtype, decode_bytes(plan, d) ? workspace : nullptr, stream);
    p.offsets = group_offsets; p.shared = shared; p.groups = groups; p.H = H;
    p.c = std::fabs(p.d.c); p.negative = scale < 0;
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
    const bool bf = cache->dtype == SAWATTN_BF16;
    if (d == 128) return bf ? launch_shared<128, true>(p, grid, stream) : launch_shared<128, false>(p, grid, stream);
    return bf ? launch_shared<64, true>(p, grid, stream) : launch_shared<64, false>(p, grid, stream);
}

}  // extern "C"
