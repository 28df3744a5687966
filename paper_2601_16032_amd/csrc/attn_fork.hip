// Requests that share pages: attn_kv_fork (which pages the requests of the next step hold), attn_kv_copy (the pages they have to copy),
// attn_kv_shared_rows (how many leading rows a group of requests has in the same pages).
//
// attn_kv_fork keeps no counts of who holds a page.  The tables say it: a page is given back if a request of the old batch holds it and none of
// the new one does, so a call marks both and compares, and there is nothing to keep up to date between calls.  With n rows and pages of
// p rows a new request takes the n / p whole pages of its source as they are.  A part-filled last page is written on, so it has one holder:
// the first request that goes on from the source's own part-filled page takes it over, all others get a fresh page and an entry in the
// list of copies.  Fresh pages are dealt out in the order of the requests, pages given back in the order of their numbers: nothing depends on timing.
//
// Bound by latency: a few numbers per request, four bytes per table entry in and out.  Three launches (numbers of requests; tables and marks; pages
// given back), each of which needs all of the one before; one where all tables together are short (kv_fork_few_kernel: 8 requests of 125 pages 4.6 us, in three
// launches 2.6 + 3.0 + 3.9).  1000 requests of up to 512 pages 4.1 + 4.2 + 4.3 us, 100 that become 4000 of up to 1024 pages 11 + 6 + 2.4.
namespace sawattn {

constexpr int kForkThreads = 1024, kForkEach = SAWATTN_MOST_REQUESTS / kForkThreads;      // requests of a thread at most
constexpr int kForkTableThreads = 256, kForkRow = 4 * kForkTableThreads;                   // table entries of a workgroup
constexpr int kForkPages = 16 * kForkThreads, kForkFreeGrid = 256;                         // pages of a workgroup at a time, 16 marks of a thread; workgroups at most (every
                                                                                           // one reads the marks in front of its own)
constexpr int kForkFewRequests = kForkThreads, kForkFewPages = 1 << 17, kForkFewEntries = 1 << 14;      // of a call that one workgroup does all of, at most

struct ForkParams {
    const int* lengths;
    const int* source;
    const int* rows;          // NULL: no bound
    const int* table;
    int* table_out;
    long long table_stride, out_stride;
    int* ring;
    const int* state;
    int* lengths_out;
    int* copies;              // [N][3]
    int* state_out;
    u4* kept;                 // workspace: a byte for every page, not 0 if a new request holds it
    u4* held;                 // ... if an old one does
    int4* plan;               // [N], ForkPlan
    int2* taken;              // (pages taken from the ring, pages that were in it)
    int R, N, max_pages, shift, pages, ring_size, mark_words;      // words of 16 marks
};

struct ForkPlan {      // of a new request
    int count;         // entries taken from its source
    int fresh;         // the fresh page's entry behind them, or -1
    int page;          // that page
    int marked;        // entries that another request of the same source marks
};

__device__ __forceinline__ int fork_length(const ForkParams& p, int s) {
    return (int)min((long long)max(p.lengths[s], 0), (long long)p.max_pages << p.shift);
}

// Where the ring begins and how much is in it, whatever is given; and a place `i` behind its first one, i at most twice its size.
struct ForkRing {
    unsigned first, size;
    int available;
    __device__ __forceinline__ ForkRing(const ForkParams& p) {
        const int first_given = p.state[0], free_given = p.state[1];
        size = (unsigned)p.ring_size;
        first = first_given >= 0 && (unsigned)first_given < size ? (unsigned)first_given : 0u;
        available = min(max(free_given, 0), p.ring_size);
    }
    __device__ __forceinline__ unsigned at(unsigned long long i) const {
        i += first;
        if (i >= size) i -= size;
        if (i >= size) i -= size;
        return (unsigned)i;
    }
};

// Sum over the threads in front of this one, and over all.
__device__ __forceinline__ int block_before(int x, int (&of_wave)[kForkThreads / 64], int& all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, upto = lanes_upto(x);
    if (lane == 63) of_wave[wave] = upto;
    __syncthreads();
    int before = upto - x;
    all = 0;
#pragma unroll
    for (int w = 0; w < kForkThreads / 64; ++w) {
        if (w < wave) before += of_wave[w];
        all += of_wave[w];
    }
    return before;
}

// What every request holds, EACH of them worked out by a thread; keep(r, plan) gets the plans.  winner, lead, counts: LDS, an entry for every old request.  Returns the pages taken.
template <int EACH, typename KEEP>
__device__ __forceinline__ int fork_requests(const ForkParams& p, const ForkRing& ring, int* winner, int* lead, int* counts, int (&of_wave)[kForkThreads / 64], KEEP&& keep) {
    const int tid = threadIdx.x, each = (p.N + kForkThreads - 1) / kForkThreads, r0 = tid * each, in_page = (1 << p.shift) - 1;
    int s[EACH], rows[EACH], length[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const bool there = i < each && r0 + i < p.N;
        s[i] = there ? p.source[r0 + i] : -1;
        rows[i] = there && p.rows ? max(p.rows[r0 + i], 0) : 0x7fffffff;
        if (s[i] >= p.R) s[i] = -1;
    }
#pragma unroll
    for (int i = 0; i < EACH; ++i) length[i] = s[i] >= 0 ? fork_length(p, s[i]) : 0;
    for (int i = tid; i < p.R; i += kForkThreads) winner[i] = lead[i] = p.N;
    __syncthreads();
    bool last[EACH];      // ends in its source's part-filled page: the first such request takes it over
    int own_s = -1, own_last = -1;      // sources of the thread's last request, and of that if it is such a one
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        rows[i] = min(rows[i], length[i]);
        last[i] = (rows[i] & in_page) && rows[i] >> p.shift == length[i] >> p.shift;
        if (i < each) {
            own_s = s[i];
            own_last = last[i] ? s[i] : -1;
        }
    }
    // (the first of neighbours with the same source speaks for them: atomics on one place go one after the other)
    int before_s = __shfl_up(own_s, 1), before_last = __shfl_up(own_last, 1);
    if ((tid & 63) == 0) before_s = before_last = -1;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (s[i] >= 0 && s[i] != before_s) atomicMin(&lead[s[i]], r0 + i);
        if (last[i] && s[i] != before_last) atomicMin(&winner[s[i]], r0 + i);
        before_s = s[i];
        before_last = last[i] ? s[i] : -1;
    }
    __syncthreads();
    int missing = 0;
    bool misses[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (last[i]) last[i] = winner[s[i]] == r0 + i;
        misses[i] = (rows[i] & in_page) && !last[i];
        missing += misses[i];
    }
    int all;
    int before = block_before(missing, of_wave, all);
    int count[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const bool ok = !misses[i] || before < ring.available;
        count[i] = ok ? (rows[i] >> p.shift) + last[i] : 0;
        before += misses[i];
        if (s[i] >= 0 && lead[s[i]] == r0 + i) counts[s[i]] = count[i];
    }
    __syncthreads();
    before -= missing;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int r = r0 + i;
        if (i >= each || r >= p.N) continue;
        const int full = rows[i] >> p.shift;
        int from = -1, to = -1;
        bool ok = true;
        if (misses[i]) {
            ok = before < ring.available;
            from = p.table[s[i] * p.table_stride + full];
            if (ok) to = p.ring[ring.at((unsigned)before)];
            ++before;
        }
        p.lengths_out[r] = ok ? rows[i] : 0;
        p.copies[3 * r] = from;
        p.copies[3 * r + 1] = to;
        p.copies[3 * r + 2] = misses[i] ? rows[i] & in_page : 0;
        keep(r, ForkPlan{count[i], misses[i] && ok ? full : -1, to, s[i] >= 0 && lead[s[i]] != r ? counts[s[i]] : 0});
    }
    return min(all, ring.available);
}

// The first workgroup works out what every request holds, the others clear the marks.
__global__ __launch_bounds__(kForkThreads) void kv_fork_kernel(ForkParams p) {
    __shared__ int winner[SAWATTN_MOST_REQUESTS], lead[SAWATTN_MOST_REQUESTS], counts[SAWATTN_MOST_REQUESTS];
    __shared__ int of_wave[kForkThreads / 64];
    const int tid = threadIdx.x;
    if (blockIdx.x) {
        for (int i = (blockIdx.x - 1) * kForkThreads + tid; i < p.mark_words; i += (gridDim.x - 1) * kForkThreads)
            p.kept[i] = p.held[i] = u4{0, 0, 0, 0};
        return;
    }
    const ForkRing ring(p);
    const int taken = fork_requests<kForkEach>(p, ring, winner, lead, counts, of_wave, [&](int r, const ForkPlan& x) { p.plan[r] = int4{x.count, x.fresh, x.page, x.marked}; });
    if (tid == 0) *p.taken = int2{taken, ring.available};
}

// Tables: a workgroup takes kForkRow entries of one request.  First the old batch's, whose pages it marks as held, then the new one's.  (What
// several workgroups mark, they mark alike; of the requests of one source mostly the first does it for all: a mark is a line of the L2 to itself, 100 prompts that become
// 4000 requests of up to 1024 pages 9.2 -> 6.2 us.)
__global__ __launch_bounds__(kForkTableThreads) void kv_fork_table_kernel(ForkParams p, int parts) {
    const int item = blockIdx.x / parts, from = (int)(blockIdx.x - item * parts) * kForkRow + threadIdx.x;
    constexpr int kEach = kForkRow / kForkTableThreads;
    const bool old = item < p.R;
    const int r = old ? item : item - p.R;
    unsigned char* const marks = reinterpret_cast<unsigned char*>(old ? p.held : p.kept);
    int s;
    int4 plan = {0, -1, 0, 0};
    if (old) {
        s = r;
        plan.x = (int)(((long long)fork_length(p, r) + (1 << p.shift) - 1) >> p.shift);
    } else {
        s = p.source[r];
        plan = p.plan[r];
    }
    const int* const row = p.table + s * p.table_stride;
    int* const out = p.table_out + r * p.out_stride;
    int page[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) page[i] = from + i * kForkTableThreads < plan.x ? row[from + i * kForkTableThreads] : -1;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int j = from + i * kForkTableThreads;
        if (j < plan.x) {
            if (j >= plan.w && (unsigned)page[i] < (unsigned)p.pages) marks[page[i]] = 1;
            if (!old) out[j] = page[i];
        }
        if (!old && j == plan.y) out[j] = plan.z;
    }
}

// Pages that were held and are no longer, by their numbers, behind the last one in the ring.  A workgroup takes `each` times kForkPages and counts those in front of its own.
__global__ __launch_bounds__(kForkThreads) void kv_fork_free_kernel(ForkParams p, int each) {
    __shared__ int of_wave[2][kForkThreads / 64];
    const int tid = threadIdx.x;
    auto freed = [&](unsigned word) {      // one bit to a byte
        u4 m = {0, 0, 0, 0};
        if (word < (unsigned)p.mark_words) m = p.held[word] & ~p.kept[word];
        return m;
    };
    auto count = [](u4 m) { return __popc(m[0]) + __popc(m[1]) + __popc(m[2]) + __popc(m[3]); };
    const unsigned chunk0 = blockIdx.x * each;
    u4 mine = freed(chunk0 * kForkThreads + tid);
    const int2 taken = *p.taken;
    const ForkRing ring(p);
    int in_front = 0;
#pragma unroll 4
    for (unsigned c = 0; c < chunk0; ++c) in_front += count(freed(c * kForkThreads + tid));
    int all;      // in front of the chunk
    block_before(in_front, of_wave[0], all);
    const int room = p.ring_size - taken.y;      // (there is room for all of them if the ring has a place for every page)
    for (unsigned chunk = chunk0;;) {
        int own;
        int before = all + block_before(count(mine), of_wave[1], own);
        if (count(mine))
#pragma unroll
            for (int w = 0; w < 4; ++w)
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (mine[w] >> (8 * b) & 1) {
                        if (before < room) p.ring[ring.at((unsigned long long)taken.y + (unsigned)before)] = (int)((chunk * kForkThreads + tid) * 16 + w * 4 + b);
                        ++before;
                    }
        all += own;
        if (++chunk == chunk0 + each) break;
        mine = freed(chunk * kForkThreads + tid);
        __syncthreads();      // of_wave has been read
    }
    if (blockIdx.x == gridDim.x - 1 && tid == 0) {
        p.state_out[0] = (int)ring.at((unsigned)taken.x);
        p.state_out[1] = taken.y - taken.x + min(all, room);
    }
}

// All of it in one workgroup, the marks in LDS, a bit to a page: for few and short tables, where the launches take longer than the work.
__global__ __launch_bounds__(kForkThreads) void kv_fork_few_kernel(ForkParams p) {
    __shared__ int winner[kForkFewRequests], lead[kForkFewRequests], counts[kForkFewRequests], of_wave[kForkThreads / 64], of_wave_freed[kForkThreads / 64];
    __shared__ ForkPlan plan[kForkFewRequests];
    extern __shared__ unsigned marks[];      // held, kept
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, words = (p.pages + 31) / 32, each = (words + kForkThreads - 1) / kForkThreads;
    unsigned* const held = marks;
    unsigned* const kept = marks + words;
    const ForkRing ring(p);
    for (int i = tid; i < 2 * words; i += kForkThreads) marks[i] = 0;
    const int taken = fork_requests<1>(p, ring, winner, lead, counts, of_wave, [&](int r, const ForkPlan& x) { plan[r] = x; });
    __syncthreads();
    for (int item = wave; item < p.R + p.N; item += kForkThreads / 64) {
        const bool old = item < p.R;
        const int r = old ? item : item - p.R;
        ForkPlan x = {0, -1, 0, 0};
        if (old) x.count = (int)(((long long)fork_length(p, r) + (1 << p.shift) - 1) >> p.shift);
        else x = plan[r];
        const int* const row = p.table + (old ? r : p.source[r]) * p.table_stride;
        int* const out = p.table_out + r * p.out_stride;
        unsigned* const bits = old ? held : kept;
#pragma unroll 4
        for (int j = lane; j < x.count; j += 64) {
            const int page = row[j];
            if (j >= x.marked && (unsigned)page < (unsigned)p.pages) atomicOr(&bits[page / 32], 1u << page % 32);
            if (!old) out[j] = page;
        }
        if (!old && lane == 0 && x.fresh >= 0) out[x.fresh] = x.page;
    }
    __syncthreads();
    int mine = 0;
    for (int i = 0; i < each; ++i) {
        const int word = tid * each + i;
        if (word < words) mine += __popc(held[word] & ~kept[word]);
    }
    int all;
    int before = block_before(mine, of_wave_freed, all);
    const int room = p.ring_size - ring.available;
    for (int i = 0; mine && i < each; ++i) {
        const int word = tid * each + i;
        for (unsigned bits = word < words ? held[word] & ~kept[word] : 0u; bits; bits &= bits - 1) {
            if (before < room) p.ring[ring.at((unsigned long long)ring.available + (unsigned)before)] = word * 32 + __builtin_ctz(bits);
            ++before;
        }
    }
    if (tid == 0) {
        p.state_out[0] = (int)ring.at((unsigned)taken);
        p.state_out[1] = ring.available - taken + min(all, room);
    }
}

// ---- copies
//
// A row of a head is d elements side by side; of a copy there are heads * rows of them in each of K and V of each layer.  They are dealt out in
// pieces of 64 rows (128 at d = 64), counted through all copies by a sum that every workgroup makes for itself (entries that are none cost nothing behind it).
// Bound by memory: 121 pages of 64 rows and fewer, 8 heads of 128, in 16 layers, 242 MB read and written, 54 us, 4.5 TB/s; loaded and stored cached 57.5.
constexpr int kCopyThreads = 256, kCopyLayers = 32, kCopyEach = SAWATTN_MOST_REQUESTS / kCopyThreads;
constexpr int kCopyAhead = 4;      // 16-byte pieces of a thread on their way

struct CopyLayer {
    char* data[2];                       // K, V
    long long page[2], head[2], row[2];      // bytes
};

struct CopyParams {
    CopyLayer layer[kCopyLayers];
    const int* copies;
    int n, layers, heads, page_size, pages;
};

template <int D>
__global__ __launch_bounds__(kCopyThreads) void kv_copy_kernel(CopyParams p) {
    constexpr int kLanes = D / 8, kRows = kCopyThreads / kLanes, kPiece = kRows * kCopyAhead;      // lanes to a row, rows at a time, rows of a piece
    __shared__ int upto[SAWATTN_MOST_REQUESTS];      // pieces of the copies up to and including this one
    __shared__ int of_wave[kCopyThreads / 64];
    const int tid = threadIdx.x, each = (p.n + kCopyThreads - 1) / kCopyThreads, i0 = tid * each;
    auto rows_of = [&](int i, int& from, int& to) {
        from = p.copies[3 * i];
        to = p.copies[3 * i + 1];
        const bool good = (unsigned)from < (unsigned)p.pages && (unsigned)to < (unsigned)p.pages && from != to;
        return good ? min(max(p.copies[3 * i + 2], 0), p.page_size) : 0;
    };
    int pieces[kCopyEach], mine = 0;
#pragma unroll
    for (int i = 0; i < kCopyEach; ++i) {
        int from, to;
        pieces[i] = i < each && i0 + i < p.n ? (rows_of(i0 + i, from, to) * p.heads + kPiece - 1) / kPiece : 0;
        mine += pieces[i];
    }
    const int lane = tid & 63, wave = tid >> 6, in_wave = lanes_upto(mine);
    if (lane == 63) of_wave[wave] = in_wave;
    __syncthreads();
    int at = in_wave - mine, total = 0;
#pragma unroll
    for (int w = 0; w < kCopyThreads / 64; ++w) {
        if (w < wave) at += of_wave[w];
        total += of_wave[w];
    }
#pragma unroll
    for (int i = 0; i < kCopyEach; ++i)
        if (i < each && i0 + i < p.n) upto[i0 + i] = at += pieces[i];
    __syncthreads();

    const long long items = (long long)total * p.layers * 2;
    for (long long item = blockIdx.x; item < items; item += gridDim.x) {
        const int tensor = (int)(item / total), piece = (int)(item - (long long)tensor * total);
        int low = 0, high = p.n - 1;
        while (low < high) {
            const int mid = (low + high) >> 1;
            if (upto[mid] > piece) high = mid; else low = mid + 1;
        }
        int from, to;
        const int rows = rows_of(low, from, to), first = (piece - (low ? upto[low - 1] : 0)) * kPiece;
        const CopyLayer& l = p.layer[tensor >> 1];
        const int v = tensor & 1;
        const char* source = l.data[v] + from * l.page[v];
        char* target = l.data[v] + to * l.page[v];
        u4 x[kCopyAhead];
        long long where[kCopyAhead];
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i) {
            const int flat = first + i * kRows + tid / kLanes, head = (unsigned)flat / (unsigned)max(rows, 1), row = flat - head * rows;
            where[i] = head < p.heads && rows ? head * l.head[v] + row * l.row[v] + tid % kLanes * 16 : -1;
            if (where[i] >= 0) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u4*>(source + where[i]));
        }
#pragma unroll
        for (int i = 0; i < kCopyAhead; ++i)
            if (where[i] >= 0) __builtin_nontemporal_store(x[i], reinterpret_cast<u4*>(target + where[i]));
    }
}

// ---- common rows
//
// A workgroup to a group; a thread to a table column and a share of the requests, at whose entries it looks, sixteen on their way at a time.  8 requests of 250 pages 4 us, 40 groups
// of 25 of up to 1024 pages 7, one of 256 requests of 260 pages 10.  A compute unit reads 14000 entries a microsecond: where groups have more than kCommonSplit of them on average, a
// first launch writes what the lengths allow and in a second one several workgroups to a group lower that (1000 requests of 512 pages 40 -> 13 us; a launch is 4).
constexpr int kCommonThreads = 1024, kCommonAhead = 16, kCommonSplit = 1 << 17, kCommonParts = 64;
enum CommonPass : int { kCommonAll, kCommonLengths, kCommonPages };

__global__ __launch_bounds__(kCommonThreads) void kv_shared_rows_kernel(const int* lengths, const int* table, long long stride, int max_pages, int shift,
                                                                      const int* offsets, int R, int* shared, int pass) {
    __shared__ int least, count, differ;
    __shared__ unsigned short there[SAWATTN_MOST_REQUESTS];      // the requests that hold a row, in any order
    const int tid = threadIdx.x, g = blockIdx.x;
    const int begin = min(max(offsets[g], 0), R), end = min(max(offsets[g + 1], 0), R);
    if (tid == 0) {
        least = 0x7fffffff;
        count = 0;
        differ = max_pages;
    }
    __syncthreads();
    for (int r = begin + tid; r < end; r += kCommonThreads) {
        const int length = lengths[r];
        if (length > 0) {
            atomicMin(&least, length);
            there[atomicAdd(&count, 1)] = (unsigned short)r;
        }
    }
    __syncthreads();
    const int n = count;
    const int pages = n ? min(least >> shift, max_pages) : 0;
    if (pass != kCommonLengths && n > 1) {
        const int part = pass == kCommonPages ? (int)((unsigned)pages / gridDim.y) + 1 : pages;
        const int first = min((int)blockIdx.y * part, pages), last = min(first + part, pages);
        // (quotients of numbers up to 1024: half of one over the divisor is more than the reciprocal is off by)
        const int across = min(max(last - first, 1), kCommonThreads);
        const float one = __builtin_amdgcn_rcpf((float)across);
        const int shares = (int)((kCommonThreads + 0.5f) * one), share = (int)(((float)tid + 0.5f) * one), column = tid - share * across;
        for (int j0 = first; j0 < last; j0 += across) {
            const int j = j0 + column;
            if (j < last && share < shares) {
                const int page = table[there[0] * stride + j];
                bool same = true;
                for (int i0 = 1 + share * kCommonAhead; i0 < n; i0 += kCommonAhead * shares) {
                    int other[kCommonAhead];
#pragma unroll
                    for (int i = 0; i < kCommonAhead; ++i) other[i] = table[there[min(i0 + i, n - 1)] * stride + j];
#pragma unroll
                    for (int i = 0; i < kCommonAhead; ++i) same = same && other[i] == page;
                }
                if (!same) atomicMin(&differ, j);
            }
            __syncthreads();
            if (differ < j0 + across) break;      // (uniform: nobody changes it before the next barrier)
            __syncthreads();
        }
    }
    if (tid == 0) {
        const int rows = min(differ, pages) << shift;
        if (pass != kCommonPages) shared[g] = rows;
        else if (differ < pages) atomicMin(shared + g, rows);
    }
}

struct ForkWorkspace {      // bytes, from the front
    size_t held, plan, taken, all;
    ForkWorkspace(int N, int pages) {
        const size_t marks = ((size_t)pages + 15) / 16 * 16;
        held = marks;
        plan = 2 * marks;
        taken = plan + sizeof(int4) * (size_t)N;
        all = taken + sizeof(int2);
    }
};

}  // namespace sawattn

extern "C" {

int attn_kv_fork_workspace_bytes(int R, int N, int pages, size_t* bytes) {
    using namespace sawattn;
    if (!bytes) return fail(SAWATTN_ERR_INVALID_ARG, "bytes must be non-null");
    if (R <= 0 || N <= 0 || pages <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "R, N and pages must be positive");
    if (R > SAWATTN_MOST_REQUESTS || N > SAWATTN_MOST_REQUESTS) return fail(SAWATTN_ERR_UNSUPPORTED, "more requests than SAWATTN_MOST_REQUESTS");
    *bytes = ForkWorkspace(N, pages).all;
    return SAWATTN_OK;
}

int attn_kv_fork(const int32_t* lengths, int R, const int32_t* source, const int32_t* rows, int N, const int32_t* table, int64_t table_stride,
                 int32_t* table_out, int64_t table_out_stride, int max_pages, int page_size, int pages, int32_t* free_pages, int ring,
                 const int32_t* free_state, int32_t* lengths_out, int32_t* copies, int32_t* free_state_out, void* workspace, size_t workspace_bytes,
                 void* hip_stream) {
    using namespace sawattn;
    size_t need = 0;
    const int rc = attn_kv_fork_workspace_bytes(R, N, pages, &need);
    if (rc != SAWATTN_OK) return rc;
    if (max_pages <= 0 || ring <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "max_pages and ring must be positive");
    if (page_shift(page_size) < 0) return fail(SAWATTN_ERR_UNSUPPORTED, "page size must be a power of two from 16 to 2^20");
    if ((long long)std::max(R, N) * max_pages >= (1LL << 31) || (long long)max_pages * page_size >= (1LL << 31))
        return fail(SAWATTN_ERR_INVALID_ARG, "R*max_pages, N*max_pages and max_pages*page_size must be below 2^31");
    if (table_stride < max_pages || table_out_stride < max_pages || (double)table_stride * R >= 1e18 || (double)table_out_stride * N >= 1e18)
        return fail(SAWATTN_ERR_INVALID_ARG, "strides of the tables must be at least max_pages");
    if (!lengths || !source || !table || !table_out || !free_pages || !free_state || !lengths_out || !copies || !free_state_out || !workspace)
        return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_fork: a pointer is null");
    uintptr_t low_bits = 0;
    for (const void* q : {(const void*)lengths, (const void*)source, (const void*)rows, (const void*)table, (const void*)table_out,
                          (const void*)free_pages, (const void*)free_state, (const void*)lengths_out, (const void*)copies, (const void*)free_state_out})
        low_bits |= (uintptr_t)q & 3u;
    if (low_bits) return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_fork: a pointer is not aligned to its elements");
    if ((uintptr_t)workspace & 15u) return fail(SAWATTN_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    if (workspace_bytes < need) return fail(SAWATTN_ERR_INVALID_ARG, "workspace is smaller than attn_kv_fork_workspace_bytes reports");
    const unsigned long long r = (unsigned long long)R, n = (unsigned long long)N;
    auto table_bytes = [&](unsigned long long count, int64_t stride) { return 4ull * ((count - 1) * (unsigned long long)stride + max_pages); };
    const Range in[] = {{lengths, 4 * r}, {source, 4 * n}, {rows, rows ? 4 * n : 0}, {table, table_bytes(r, table_stride)}, {free_state, 8}};
    const Range out[] = {{table_out, table_bytes(n, table_out_stride)}, {free_pages, 4ull * ring}, {lengths_out, 4 * n}, {copies, 12 * n},
                         {free_state_out, 8}, {workspace, need}};
    for (const Range& o : out) {
        for (const Range& i : in)
            if (o.meets(i)) return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_fork: an output overlaps an input");
        for (const Range& other : out)
            if (&o != &other && o.meets(other)) return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_fork: two outputs overlap");
    }
    const ForkWorkspace at(N, pages);
    char* const w = static_cast<char*>(workspace);
    ForkParams p = {lengths, source, rows, table, table_out, table_stride, table_out_stride, free_pages, free_state, lengths_out, copies, free_state_out,
                    reinterpret_cast<u4*>(w), reinterpret_cast<u4*>(w + at.held), reinterpret_cast<int4*>(w + at.plan), reinterpret_cast<int2*>(w + at.taken),
                    R, N, max_pages, page_shift(page_size), pages, ring, (int)(((long long)pages + 15) / 16)};
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    if (R <= kForkFewRequests && N <= kForkFewRequests && pages <= kForkFewPages && (long long)(R + N) * max_pages <= kForkFewEntries) {
        const int words = (pages + 31) / 32;
        hipLaunchKernelGGL(kv_fork_few_kernel, dim3(1), dim3(kForkThreads), 2 * words * sizeof(unsigned), stream, p);
        return launched("attn_kv_fork");
    }
    const int clearing = std::min(255, (p.mark_words + kForkThreads - 1) / kForkThreads);
    hipLaunchKernelGGL(kv_fork_kernel, dim3(1 + clearing), dim3(kForkThreads), 0, stream, p);
    int status = launched("attn_kv_fork");
    if (status != SAWATTN_OK) return status;
    const int parts = (int)(((long long)max_pages + kForkRow - 1) / kForkRow);
    hipLaunchKernelGGL(kv_fork_table_kernel, dim3((R + N) * parts), dim3(kForkTableThreads), 0, stream, p, parts);      // (below 2^22 + 2^13)
    status = launched("attn_kv_fork");
    if (status != SAWATTN_OK) return status;
    const int chunks = (int)(((long long)pages + kForkPages - 1) / kForkPages), each = (chunks + kForkFreeGrid - 1) / kForkFreeGrid;
    hipLaunchKernelGGL(kv_fork_free_kernel, dim3((chunks + each - 1) / each), dim3(kForkThreads), 0, stream, p, each);
    return launched("attn_kv_fork");
}

int attn_kv_copy(const sawattn_kv_cache* caches, int layers, const int32_t* copies, int n, void* hip_stream) {
    using namespace sawattn;
    if (layers <= 0 || n <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "layers and n must be positive");
    if (!caches || !copies) return fail(SAWATTN_ERR_INVALID_ARG, "caches and copies must be non-null");
    if (n > SAWATTN_MOST_REQUESTS) return fail(SAWATTN_ERR_UNSUPPORTED, "more copies than SAWATTN_MOST_REQUESTS");
    if ((uintptr_t)copies & 3u) return fail(SAWATTN_ERR_INVALID_ARG, "copies must be 4-byte aligned");
    const sawattn_kv_cache& one = caches[0];
    for (int l = 0; l < layers; ++l) {
        const sawattn_kv_cache& c = caches[l];
        const int rc = check_cache(&c, true);
        if (rc != SAWATTN_OK) return rc;
        if (c.pages != one.pages || c.page_size != one.page_size || c.heads != one.heads || c.d != one.d || c.dtype != one.dtype)
            return fail(SAWATTN_ERR_INVALID_ARG, "caches must share pages, page_size, heads, d and dtype");
    }
    if ((long long)n * one.heads * one.page_size >= (1LL << 31) - 128)      // (rows are counted in 32 bits, rounded up to pieces of 64 or 128)
        return fail(SAWATTN_ERR_INVALID_ARG, "n*heads*page_size must be below 2^31 - 128");
    const Range list(copies, 12ull * n);
    auto extent = [](int count, int64_t stride) { return count > 1 ? (unsigned long long)(count - 1) * stride : 0ull; };
    for (int l = 0; l < layers; ++l) {
        const sawattn_kv_cache& c = caches[l];
        const Range k(c.k, 2 * (extent(c.pages, c.k_page) + extent(c.heads, c.k_head) + extent(c.page_size, c.k_row) + c.d));
        const Range v(c.v, 2 * (extent(c.pages, c.v_page) + extent(c.heads, c.v_head) + extent(c.page_size, c.v_row) + c.d));
        if (list.meets(k) || list.meets(v)) return fail(SAWATTN_ERR_INVALID_ARG, "copies must not lie in a cache");
    }
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    const int piece = kCopyThreads / (one.d / 8) * kCopyAhead;
    const double pieces = (double)n * (((double)one.heads * one.page_size + piece - 1) / piece);
    for (int l0 = 0; l0 < layers; l0 += kCopyLayers) {
        CopyParams p{};
        p.layers = std::min(kCopyLayers, layers - l0);
        for (int l = 0; l < p.layers; ++l) {
            const sawattn_kv_cache& c = caches[l0 + l];
            p.layer[l] = {{static_cast<char*>(c.k), static_cast<char*>(c.v)}, {2 * c.k_page, 2 * c.v_page}, {2 * c.k_head, 2 * c.v_head}, {2 * c.k_row, 2 * c.v_row}};
        }
        p.copies = copies; p.n = n; p.heads = one.heads; p.page_size = one.page_size; p.pages = one.pages;
        const int grid = (int)std::min(2048.0, std::max(1.0, pieces * p.layers * 2));
        if (one.d == 128) hipLaunchKernelGGL((kv_copy_kernel<128>), dim3(grid), dim3(kCopyThreads), 0, stream, p);
        else hipLaunchKernelGGL((kv_copy_kernel<64>), dim3(grid), dim3(kCopyThreads), 0, stream, p);
        const int rc = launched("attn_kv_copy");
        if (rc != SAWATTN_OK) return rc;
    }
    return SAWATTN_OK;
}

int attn_kv_shared_rows(const int32_t* lengths, int R, const int32_t* table, int64_t table_stride, int max_pages, int page_size, const int32_t* group_offsets,
                        int groups, int32_t* shared, void* hip_stream) {
    using namespace sawattn;
    if (R <= 0 || max_pages <= 0 || groups <= 0) return fail(SAWATTN_ERR_INVALID_ARG, "R, max_pages and groups must be positive");
    if (R > SAWATTN_MOST_REQUESTS || groups > SAWATTN_MOST_REQUESTS) return fail(SAWATTN_ERR_UNSUPPORTED, "more requests or groups than SAWATTN_MOST_REQUESTS");
    if (page_shift(page_size) < 0) return fail(SAWATTN_ERR_UNSUPPORTED, "page size must be a power of two from 16 to 2^20");
    if ((long long)max_pages * page_size >= (1LL << 31)) return fail(SAWATTN_ERR_INVALID_ARG, "max_pages*page_size must be below 2^31");
    if (table_stride < max_pages || (double)table_stride * R >= 1e18) return fail(SAWATTN_ERR_INVALID_ARG, "table_stride must be at least max_pages");
    if (!lengths || !table || !group_offsets || !shared) return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_shared_rows: a pointer is null");
    if (((uintptr_t)lengths | (uintptr_t)table | (uintptr_t)group_offsets | (uintptr_t)shared) & 3u)
        return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_shared_rows: a pointer is not aligned to its elements");
    const Range out(shared, 4ull * groups);
    for (const Range& i : {Range(lengths, 4ull * R), Range(table, 4ull * ((unsigned long long)(R - 1) * table_stride + max_pages)), Range(group_offsets, 4ull * (groups + 1))})
        if (out.meets(i)) return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_shared_rows: an output overlaps an input");
    hipStream_t stream = static_cast<hipStream_t>(hip_stream);
    auto launch = [&](int parts, CommonPass pass) {
        hipLaunchKernelGGL(kv_shared_rows_kernel, dim3(groups, parts), dim3(kCommonThreads), 0, stream, lengths, table, (long long)table_stride, max_pages,
                           page_shift(page_size), group_offsets, R, shared, (int)pass);
    };
    const long long each = (long long)R * max_pages / groups;      // entries of a group
    if (each <= kCommonSplit) {
        launch(1, kCommonAll);
    } else {
        launch(1, kCommonLengths);
        const int status = launched("attn_kv_shared_rows");
        if (status != SAWATTN_OK) return status;
        launch((int)std::min<long long>(each / (kCommonSplit / 8) + 1, kCommonParts), kCommonPages);
    }
    return launched("attn_kv_shared_rows");
}

}  // extern "C"
