// attn_kv_pages: page tables and slot maps from request lengths.
//
// Three sums over the requests, in order, decide everything: of their tokens, of the pages they miss and of the pages they give back.
// With the sums upto and including request r written T_r, P_r and Q_r: r gets its rows if they fit its table row, P_r <= pages free
// and T_r <= tokens of the batch.  P and T never fall, so what is left over is a tail of the requests that need pages, and the pages
// taken are the largest P_r granted.  Token t belongs to the first r with T_r > t; its row is length_r + t - T_(r-1).
//
// Every workgroup makes the sums for itself (4096 requests at most, 4 of a thread, one scan over the threads; from the L2) and then takes
// its share of the tokens, each found by bisection in LDS: one launch, no workspace, nothing to wait for.  The pages need no loop of their own:
// every new page has exactly one token whose row is its first, and that token enters it into the table.
namespace sawattn {

constexpr int kPagesEach = 4;      // requests of a thread at most

struct PagesParams {
    const int* lengths;
    const int* added;
    int* table;
    long long table_stride;
    int* ring;
    const int* state;
    int* lengths_out;
    int* granted;
    int* offsets;
    int* state_out;
    long long* slots;
    int* positions;
    int R, max_pages, shift, ring_size, tokens;
};

struct PageSums {      // over requests
    long long tokens;
    int missing, back;
    __device__ __forceinline__ void add(const PageSums& o) { tokens += o.tokens; missing += o.missing; back += o.back; }
};

struct PageRequest {
    int length, added;      // added < 0: ends
    int held, missing, back;
    bool fits;
    __device__ __forceinline__ PageRequest() {}
    __device__ __forceinline__ PageRequest(const PagesParams& p, int given, int new_tokens) {
        length = max(given, 0);
        added = new_tokens;
        const long long most = (long long)p.max_pages << p.shift, end = (long long)length + max(added, 0);
        const int round = (1 << p.shift) - 1;
        held = (int)(((long long)length + round) >> p.shift);
        fits = added > 0 && end <= most;
        missing = fits ? (int)((end + round) >> p.shift) - held : 0;
        back = added < 0 ? min(held, p.max_pages) : 0;
    }
    __device__ __forceinline__ PageSums sums() const { return {(long long)max(added, 0), missing, back}; }
};

// THREADS: 256, or 1024 for more than 1024 requests, which leaves a thread four at most (257 requests with 256 threads 4.2 us, with 1024 4.6).
template <int THREADS>
__global__ __launch_bounds__(THREADS) void kv_pages_kernel(PagesParams p) {
    __shared__ int tokens_upto[SAWATTN_MOST_REQUESTS];      // T_r
    __shared__ int back_upto[SAWATTN_MOST_REQUESTS];        // Q_r
    __shared__ int first_page[SAWATTN_MOST_REQUESTS];       // P_(r-1): its first new page, counted from the ring's first; -1: nothing granted
    __shared__ int length_of[SAWATTN_MOST_REQUESTS];
    __shared__ PageSums of_wave[THREADS / 64];
    __shared__ int taken_by_wave[THREADS / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const unsigned F = (unsigned)p.ring_size;
    const int first_given = p.state[0], free_given = p.state[1];
    const int each = (p.R + THREADS - 1) / THREADS, r0 = tid * each;

    // the thread's requests: all of their numbers on their way at once (and none read twice)
    PageRequest request[kPagesEach];
    int given[kPagesEach], added[kPagesEach];
#pragma unroll
    for (int i = 0; i < kPagesEach; ++i) {
        const bool there = i < each && r0 + i < p.R;
        given[i] = there ? p.lengths[r0 + i] : 0;
        added[i] = there ? p.added[r0 + i] : 0;
    }
    PageSums mine = {0, 0, 0};
#pragma unroll
    for (int i = 0; i < kPagesEach; ++i) {
        request[i] = PageRequest(p, given[i], added[i]);
        mine.add(request[i].sums());
    }
    const PageSums upto = {lanes_upto(mine.tokens), lanes_upto(mine.missing), lanes_upto(mine.back)};
    if (lane == 63) of_wave[wave] = upto;
    __syncthreads();
    PageSums before = {upto.tokens - mine.tokens, upto.missing - mine.missing, upto.back - mine.back}, all = {0, 0, 0};
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        if (w < wave) before.add(of_wave[w]);
        all.add(of_wave[w]);
    }

    // the ring's state: whatever is there, indexes stay inside
    const unsigned first = first_given >= 0 && (unsigned)first_given < F ? (unsigned)first_given : 0u;
    const int available = min(max(free_given, 0), p.ring_size);
    int taken = 0;
#pragma unroll
    for (int i = 0; i < kPagesEach; ++i) {
        const int r = r0 + i;
        if (i >= each || r >= p.R) continue;
        const PageRequest& q = request[i];
        PageSums with = before;
        with.add(q.sums());
        const bool there = with.missing <= available && with.tokens <= p.tokens;
        const bool ok = q.fits && with.tokens <= p.tokens && (q.missing == 0 || with.missing <= available);
        if (there) taken = max(taken, with.missing);
        const int T = (int)min(with.tokens, 0x7fffffffLL);
        tokens_upto[r] = T;
        back_upto[r] = with.back;
        first_page[r] = ok ? before.missing : -1;
        length_of[r] = q.length;
        if (blockIdx.x == 0) {
            p.lengths_out[r] = q.added < 0 ? 0 : ok ? q.length + q.added : q.length;
            p.granted[r] = ok ? q.added : 0;
            p.offsets[r + 1] = T;
        }
        before = with;
    }
    if (blockIdx.x == 0) {
#pragma unroll
        for (int step = 1; step < 64; step *= 2) taken = max(taken, __shfl_xor(taken, step));
        if (lane == 0) taken_by_wave[wave] = taken;
    }
    __syncthreads();
    if (blockIdx.x == 0 && tid == 0) {
        for (int w = 0; w < THREADS / 64; ++w) taken = max(taken, taken_by_wave[w]);
        p.offsets[0] = 0;
        p.state_out[0] = (int)(((unsigned long long)first + (unsigned)taken) % F);
        p.state_out[1] = min(available - taken + all.back, p.ring_size);
    }

    const int stride = gridDim.x * THREADS;
    const int filled = (int)min(all.tokens, (long long)p.tokens);
    for (int t = blockIdx.x * THREADS + tid; t < p.tokens; t += stride) {
        long long slot = -1;
        int row = -1;
        if (t < filled) {
            int low = 0, high = p.R - 1;
            while (low < high) {
                const int mid = (low + high) >> 1;
                if (tokens_upto[mid] > t) high = mid; else low = mid + 1;
            }
            if (first_page[low] >= 0) {
                const int length = length_of[low];
                row = length + t - (low ? tokens_upto[low - 1] : 0);
                const int index = row >> p.shift, new_index = index - (int)(((long long)length + (1 << p.shift) - 1) >> p.shift);
                int* entry = p.table + low * p.table_stride + index;
                int page;
                if (new_index >= 0) {
                    unsigned at = first + (unsigned)(first_page[low] + new_index);      // (below 2 F)
                    if (at >= F) at -= F;
                    page = p.ring[at];
                    if ((row & ((1 << p.shift) - 1)) == 0) *entry = page;
                } else {
                    page = *entry;
                }
                slot = ((long long)page << p.shift) + (row & ((1 << p.shift) - 1));
            }
        }
        p.slots[t] = slot;
        p.positions[t] = row;
    }
    for (int e = blockIdx.x * THREADS + tid; e < all.back; e += stride) {      // pages given back, behind the last free one
        int low = 0, high = p.R - 1;
        while (low < high) {
            const int mid = (low + high) >> 1;
            if (back_upto[mid] > e) high = mid; else low = mid + 1;
        }
        const int j = e - (low ? back_upto[low - 1] : 0);
        p.ring[((unsigned long long)first + (unsigned)available + (unsigned)e) % F] = p.table[low * p.table_stride + j];
    }
}

}  // namespace sawattn

extern "C" int attn_kv_pages(const int32_t* lengths, const int32_t* new_tokens, int R, int32_t* table, int64_t table_stride,
                             int max_pages, int page_size, int32_t* free_pages, int ring, const int32_t* free_state,
                             int32_t* lengths_out, int32_t* granted, int32_t* token_offsets, int32_t* free_state_out,
                             int64_t* slots, int32_t* positions, int tokens, void* hip_stream) {
    using namespace sawattn;
    if (R <= 0 || max_pages <= 0 || ring <= 0 || tokens < 0)
        return fail(SAWATTN_ERR_INVALID_ARG, "R, max_pages and ring must be positive, tokens not negative");
    if (R > SAWATTN_MOST_REQUESTS) return fail(SAWATTN_ERR_UNSUPPORTED, "more requests than SAWATTN_MOST_REQUESTS");
    if (page_shift(page_size) < 0) return fail(SAWATTN_ERR_UNSUPPORTED, "page size must be a power of two from 16 to 2^20");
    if ((long long)R * max_pages >= (1LL << 31) || (long long)max_pages * page_size >= (1LL << 31) ||
        tokens >= (1LL << 31) - (1 << 20))
        return fail(SAWATTN_ERR_INVALID_ARG, "R*max_pages and max_pages*page_size must be below 2^31, tokens below 2^31 - 2^20");
    if (table_stride < max_pages || (double)table_stride * R >= 1e18)
        return fail(SAWATTN_ERR_INVALID_ARG, "table_stride must be at least max_pages");
    if (!lengths || !new_tokens || !table || !free_pages || !free_state || !lengths_out || !granted || !token_offsets ||
        !free_state_out || (tokens && (!slots || !positions)))
        return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_pages: a pointer is null");
    uintptr_t low_bits = (uintptr_t)slots & 7u;
    for (const void* q : {(const void*)lengths, (const void*)new_tokens, (const void*)table, (const void*)free_pages,
                          (const void*)free_state, (const void*)lengths_out, (const void*)granted, (const void*)token_offsets,
                          (const void*)free_state_out, (const void*)positions})
        low_bits |= (uintptr_t)q & 3u;
    if (low_bits) return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_pages: a pointer is not aligned to its elements");
    const unsigned long long n = (unsigned long long)R, rows = 4ull * ((n - 1) * (unsigned long long)table_stride + max_pages);
    const Range in[] = {{lengths, 4 * n}, {new_tokens, 4 * n}, {free_state, 8}};
    const Range out[] = {{table, rows}, {free_pages, 4ull * ring}, {lengths_out, 4 * n}, {granted, 4 * n},
                         {token_offsets, 4 * n + 4}, {free_state_out, 8}, {slots, 8ull * tokens}, {positions, 4ull * tokens}};
    for (const Range& o : out) {
        for (const Range& i : in)
            if (o.meets(i)) return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_pages: an output overlaps an input");
        for (const Range& other : out)
            if (&o != &other && o.meets(other)) return fail(SAWATTN_ERR_INVALID_ARG, "attn_kv_pages: two outputs overlap");
    }
    PagesParams p = {lengths, new_tokens, table, table_stride, free_pages, free_state, lengths_out, granted, token_offsets,
                     free_state_out, reinterpret_cast<long long*>(slots), positions, R, max_pages, page_shift(page_size), ring, tokens};
    // 512 tokens to a workgroup, and a workgroup for every 64 requests at least, whose pages it may have to give back.
    const int grid = std::min(256, std::max((tokens + 511) / 512, (R + 63) / 64));
    static_assert(1024 * kPagesEach >= SAWATTN_MOST_REQUESTS, "a thread's requests");
    if (R <= 256 * kPagesEach) hipLaunchKernelGGL((kv_pages_kernel<256>), dim3(grid), dim3(256), 0, static_cast<hipStream_t>(hip_stream), p);
    else hipLaunchKernelGGL((kv_pages_kernel<1024>), dim3(grid), dim3(1024), 0, static_cast<hipStream_t>(hip_stream), p);
    return launched("attn_kv_pages");
}
