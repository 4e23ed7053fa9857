// Pages of the 4-bit cache: forking, reserving (copy on write), rolling back, bringing together.
//
// The state is a table of page ids per request, the requests' lengths and how many places of the table every page holds (its count).  Which
// page is free is its count alone, and the free page that is taken is always the lowest one, so the state after a call depends on nothing but the
// state before it: counts change by whole-number atomics whose order cannot show, and nothing is a stack.
//
//  reserve   the k-th page needed (requests in order) is the k-th lowest free one.  Pools of up to 65536 pages and 1024 requests: one
//            workgroup ranks and hands out (reserve_small_kernel).  Larger: counts per block of pages and needs per request
//            (count_kernel), ranks from both (free_kernel), then every request takes its own (take_kernel).
//  compact   n pages are in use; those behind place n (movers, in order) take the free places in front of it (holes, in order).  Ranks
//            likewise, by one workgroup (movers_small_kernel) or two launches.
//
// What bounds them: launches and chains of loads (a few microseconds each) for the whole numbers, memory for the pages themselves, whose copies share out
// pieces of 16 KB over the chip.
#include "../../include/ralm.h"
#include "ralm_common.h"
#include "kv_kernels.h"

namespace ralm {

namespace {

constexpr int COPY_PIECE = 16384;   // bytes of a page that a workgroup copies at a time
constexpr int COPY_GROUPS = 2048;   // workgroups of a copy whose number of pages is on the device

// scratch, in 32-bit words: [0, 1] the pairs of a copy; counts of free pages per block of pages; needs per block of requests; need
// of every request; the free pages in order (reserve), or the movers' places, holes, movers and movers' counts (compact); pairs of a copy
struct Scratch {
    int32_t *n_pairs, *block_free, *block_need, *need, *list, *pairs;
    int n_blocks, n_groups;
};
__host__ __device__ inline Scratch carve(int32_t *s, int64_t n_pages, int64_t R)
{
    Scratch c;
    c.n_blocks = (int)((n_pages + KV_COUNT_PAGES - 1) / KV_COUNT_PAGES);
    c.n_groups = (int)((R + KV_COUNT_REQUESTS - 1) / KV_COUNT_REQUESTS);
    c.n_pairs = s;
    c.block_free = s + 4;
    c.block_need = c.block_free + c.n_blocks;
    c.need = c.block_need + c.n_groups;
    c.list = c.need + R;
    c.pairs = c.list + 3 * n_pages;
    return c;
}

__device__ __forceinline__ int wave_sum(int v)
{
    v += (int)lane_xor<1>(v);
    v += (int)lane_xor<2>(v);
    v += (int)lane_xor<4>(v);
    v += (int)lane_xor<8>(v);
    v += (int)lane_xor<16>(v);
    v += (int)lane_xor<32>(v);
    return v;
}
// the sum of v over the workgroup's NT threads, for all of them; red: [NT / 64]
template <int NT>
__device__ __forceinline__ int group_sum(int v, int *red)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    int t = 0;
    for (int w = 0; w < NT / 64; ++w) t += red[w];
    return t;
}
// the sum of v over the threads in front of this one
template <int NT>
__device__ __forceinline__ int sum_before(int v, int *red)
{
    const int lane = threadIdx.x & 63;
    int incl = v;
    for (int s = 1; s < 64; s <<= 1) {
        const int up = __shfl_up(incl, s, 64);
        if (lane >= s) incl += up;
    }
    __syncthreads();
    if (lane == 63) red[threadIdx.x >> 6] = incl;
    __syncthreads();
    int t = 0;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) t += red[w];
    return t + incl - v;
}

constexpr int NEED_COPY = 1 << 30;   // of a request's need: the last page is copied
__device__ __forceinline__ int64_t clamped_len(int32_t len, int64_t most) { return len < 0 ? 0 : len > most ? most : len; }

// pages that request r needs for grow more tokens; more than its row of the table takes: -1
__device__ int need_of(const KvPages &kv, const int32_t *grow, int64_t r)
{
    const int T = kv.page_tokens;
    const int64_t most = (int64_t)kv.max_pages * T;
    const int64_t len = clamped_len(kv.lens[r], most), more = grow[r] < 0 ? 0 : grow[r];
    if (more == 0) return 0;
    if (len + more > most) return -1;
    const int64_t have = (len + T - 1) / T, want = (len + more + T - 1) / T;
    int need = (int)(want - have);
    if (len % T) {
        const int32_t last = kv.table[r * kv.max_pages + have - 1];
        if (last >= 0 && last < kv.n_pages && kv.refs[last] > 1) need = (need + 1) | NEED_COPY;
    }
    return need;
}

// workgroups 0 .. n_blocks-1: free pages of a block of pages; the rest: needs of a block of requests
__global__ __launch_bounds__(256) void count_kernel(KvPages kv, const int32_t *grow, int32_t *scratch)
{
    __shared__ int red[4];
    const Scratch s = carve(scratch, kv.n_pages, kv.R);
    if ((int)blockIdx.x < s.n_blocks) {
        const int64_t base = (int64_t)blockIdx.x * KV_COUNT_PAGES;
        int n = 0;
        for (int i = threadIdx.x; i < KV_COUNT_PAGES; i += 256)
            if (base + i < kv.n_pages) n += kv.refs[base + i] <= 0;
        n = group_sum<256>(n, red);
        if (threadIdx.x == 0) {
            s.block_free[blockIdx.x] = n;
            if (blockIdx.x == 0) s.n_pairs[0] = 0;
        }
        return;
    }
    const int g = (int)blockIdx.x - s.n_blocks;
    const int64_t r = (int64_t)g * KV_COUNT_REQUESTS + threadIdx.x;
    int need = 0;
    if (r < kv.R) {
        need = need_of(kv, grow, r);
        s.need[r] = need;
        need = need < 0 ? 0 : need & ~NEED_COPY;
    }
    need = group_sum<256>(need, red);
    if (threadIdx.x == 0) s.block_need[g] = need;
}

// list[k] = the k-th lowest free page, as far as pages are needed
__global__ __launch_bounds__(256) void free_kernel(KvPages kv, int32_t *scratch)
{
    __shared__ int red[4];
    const Scratch s = carve(scratch, kv.n_pages, kv.R);
    int before = 0, wanted = 0;
    for (int b = threadIdx.x; b < (int)blockIdx.x; b += 256) before += s.block_free[b];
    for (int g = threadIdx.x; g < s.n_groups; g += 256) wanted += s.block_need[g];
    before = group_sum<256>(before, red);
    wanted = group_sum<256>(wanted, red);
    if (before >= wanted) return;
    // sixteen neighbouring pages per thread
    constexpr int PER = KV_COUNT_PAGES / 256;
    const int64_t base = (int64_t)blockIdx.x * KV_COUNT_PAGES + threadIdx.x * PER;
    uint32_t free_bits = 0;
    for (int i = 0; i < PER; ++i)
        if (base + i < kv.n_pages && kv.refs[base + i] <= 0) free_bits |= 1u << i;
    int rank = before + sum_before<256>(__popc(free_bits), red);
    for (; free_bits && rank < wanted; free_bits &= free_bits - 1, ++rank) s.list[rank] = (int32_t)(base + __builtin_ctz(free_bits));
}

// a wave per request: its new pages into the table, their counts, its length; copies are put on the list
__global__ __launch_bounds__(256) void take_kernel(KvPages kv, const int32_t *grow, int32_t *granted, int32_t *scratch)
{
    const Scratch s = carve(scratch, kv.n_pages, kv.R);
    const int lane = threadIdx.x & 63;
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= kv.R) return;
    int before = 0, n_free = 0;
    const int64_t g = r / KV_COUNT_REQUESTS;
    for (int64_t i = lane; i < g; i += 64) before += s.block_need[i];
    for (int64_t i = g * KV_COUNT_REQUESTS + lane; i < r; i += 64) before += s.need[i] < 0 ? 0 : s.need[i] & ~NEED_COPY;
    for (int b = lane; b < s.n_blocks; b += 64) n_free += s.block_free[b];
    before = wave_sum(before);
    n_free = wave_sum(n_free);
    const int word = s.need[r];
    const int need = word < 0 ? 0 : word & ~NEED_COPY;
    const bool ok = word >= 0 && (need == 0 || (int64_t)before + need <= n_free);
    if (lane == 0 && granted) granted[r] = ok;
    if (!ok || grow[r] <= 0) return;
    const int T = kv.page_tokens;
    const int64_t len = clamped_len(kv.lens[r], (int64_t)kv.max_pages * T);
    const int64_t have = (len + T - 1) / T;
    const bool copy = word & NEED_COPY;
    int32_t *row = kv.table + r * kv.max_pages;
    for (int i = lane; i < need; i += 64) {
        const int32_t page = s.list[before + i];
        int64_t at = have + i - copy;
        if (copy && i == 0) {
            const int32_t old = row[at];
            const int k = atomicAdd(s.n_pairs, 1);   // copies do not depend on each other: any order of the list will do
            s.pairs[2 * k] = old;
            s.pairs[2 * k + 1] = page;
            atomicSub(&kv.refs[old], 1);
        }
        kv.refs[page] = 1;
        row[at] = page;
    }
    if (lane == 0) kv.lens[r] = (int32_t)(len + grow[r]);
}

// The same by one workgroup of 1024 threads: a request per thread, and 64 neighbouring pages, whose free ones a wave's vote makes a word of.  What bounds it are loads
// that follow from each other: lengths, last pages, their counts, the list, the table.
constexpr int SMALL_PAGES = 65536, SMALL_REQUESTS = 1024;
// words[i]: which of the pages 64 i .. 64 i + 63 are free (as far as there are pages); sixteen counts' loads under way at once, `between` is done while the first of them
// are.  A barrier follows
template <class F>
__device__ __forceinline__ void free_words(const KvPages &kv, u64 *words, F between)
{
    const int tid = threadIdx.x;
    for (int at = 0; at < kv.n_pages; at += 16384) {
        int c[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) c[i] = at + i * 1024 + tid < kv.n_pages ? kv.refs[at + i * 1024 + tid] : 1;
        if (at == 0) between();
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const u64 bits = __ballot(c[i] <= 0);
            if ((tid & 63) == 0) words[(at + i * 1024 + tid) >> 6] = bits;
        }
    }
}
// the sums of v's two halves over the threads in front of this one, and over all 1024
__device__ __forceinline__ u64 pair_before(u64 v, u64 *red, u64 &total)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    u64 incl = v;
    for (int s = 1; s < 64; s <<= 1) {
        const u64 up = (u64)(uint32_t)__shfl_up((int)(uint32_t)(incl >> 32), s, 64) << 32 | (uint32_t)__shfl_up((int)(uint32_t)incl, s, 64);
        if (lane >= s) incl += up;
    }
    if (lane == 63) red[wave] = incl;
    __syncthreads();
    u64 before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) {
        before += w < wave ? red[w] : 0;
        total += red[w];
    }
    return before + incl - v;
}
__global__ __launch_bounds__(1024) void reserve_small_kernel(KvPages kv, const int32_t *grow, int32_t *granted, int32_t *scratch)
{
    __shared__ u64 red[16], words[SMALL_PAGES / 64];
    __shared__ int prefix[SMALL_PAGES / 64], s_first[SMALL_REQUESTS], s_place[SMALL_REQUESTS], n_pairs, s_taken;
    const Scratch s = carve(scratch, kv.n_pages, kv.R);
    const int r = threadIdx.x;
    if (r == 0) n_pairs = s_taken = 0;
    int word = 0;
    free_words(kv, words, [&] { word = r < kv.R ? need_of(kv, grow, r) : 0; });
    __syncthreads();
    const int need = word < 0 ? 0 : word & ~NEED_COPY;
    u64 total;
    const u64 before = pair_before((u64)(r * 64 < kv.n_pages ? __popcll(words[r]) : 0) << 32 | (uint32_t)need, red, total);
    const int n_free = (int)(total >> 32), wanted = (int)(uint32_t)total, first = (int)(uint32_t)before;
    prefix[r] = (int)(before >> 32);
    const bool ok = word >= 0 && (need == 0 || first + need <= n_free);
    if (ok && need) atomicMax(&s_taken, first + need);   // requests that are served come first, but for those that need nothing
    const bool copy = word >= 0 && (word & NEED_COPY);
    const int T = kv.page_tokens;
    int64_t len = 0;
    if (r < kv.R) len = clamped_len(kv.lens[r], (int64_t)kv.max_pages * T);
    s_first[r] = first;
    s_place[r] = (int)((len + T - 1) / T) * 2 - (copy ? 1 : 0);   // place behind the last page; odd: the page in front of it is copied
    __syncthreads();
    for (int id = r; id < kv.n_pages && prefix[(id - r) >> 6] < wanted; id += 1024) {
        const u64 bits = words[id >> 6];
        const int rank = prefix[id >> 6] + __popcll(bits & ((1ull << (id & 63)) - 1ull));
        if ((bits >> (id & 63) & 1u) && rank < wanted) s.list[rank] = id;
    }
    __syncthreads();
    const int taken = s_taken;
    for (int i = threadIdx.x; i < taken; i += 1024) {
        // the last request whose first page is not behind page i is the one that needs it
        int lo = 0, hi = kv.R - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (s_first[mid] <= i) lo = mid;
            else hi = mid - 1;
        }
        const int32_t page = s.list[i];
        const int place = s_place[lo], nth = i - s_first[lo];
        int32_t *at = kv.table + (int64_t)lo * kv.max_pages + (place >> 1) + nth;
        if ((place & 1) && nth == 0) {
            const int32_t old = *at;
            const int k = atomicAdd(&n_pairs, 1);   // copies do not depend on each other: any order of the list will do
            s.pairs[2 * k] = old;
            s.pairs[2 * k + 1] = page;
            atomicSub(&kv.refs[old], 1);
        }
        kv.refs[page] = 1;
        *at = page;
    }
    if (r < kv.R) {
        if (granted) granted[r] = ok;
        if (ok && grow[r] > 0) kv.lens[r] = (int32_t)(len + grow[r]);
    }
    __syncthreads();
    if (r == 0) *s.n_pairs = n_pairs;
}

__device__ __forceinline__ void copy_piece(uint8_t *pages, int64_t page_bytes, int32_t n_pages, int32_t src, int32_t dst, int64_t piece)
{
    if (src < 0 || src >= n_pages || dst < 0 || dst >= n_pages || src == dst) return;
    const int64_t at = piece * COPY_PIECE;
    const int n = (int)(page_bytes - at < COPY_PIECE ? page_bytes - at : COPY_PIECE) / 16;
    const uint4 *a = reinterpret_cast<const uint4 *>(pages + src * page_bytes + at);
    uint4 *b = reinterpret_cast<uint4 *>(pages + dst * page_bytes + at);
    uint4 x[COPY_PIECE / 16 / 256];
#pragma unroll
    for (int i = 0; i < COPY_PIECE / 16 / 256; ++i)
        if ((int)threadIdx.x + 256 * i < n) x[i] = a[threadIdx.x + 256 * i];
#pragma unroll
    for (int i = 0; i < COPY_PIECE / 16 / 256; ++i)
        if ((int)threadIdx.x + 256 * i < n) b[threadIdx.x + 256 * i] = x[i];
}

// pages src -> dst: pair i at src[i * step], dst[i * step]; n pairs, or *n_dev
__global__ __launch_bounds__(256) void copy_kernel(uint8_t *pages, int64_t page_bytes, int32_t n_pages, const int32_t *src, const int32_t *dst,
                                                   int step, int64_t n, const int32_t *n_dev)
{
    if (n_dev) n = *n_dev;
    const int64_t pieces = (page_bytes + COPY_PIECE - 1) / COPY_PIECE;
    for (int64_t i = blockIdx.x; i < n * pieces; i += gridDim.x)
        copy_piece(pages, page_bytes, n_pages, src[i / pieces * step], dst[i / pieces * step], i % pieces);
}

// a wave per pair of requests
__global__ __launch_bounds__(256) void fork_kernel(KvPages kv, const int32_t *src, const int32_t *dst, const int32_t *keep, int64_t n)
{
    const int64_t i = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (i >= n) return;
    const int32_t a = src[i], b = dst[i];
    if (a < 0 || a >= kv.R || b < 0 || b >= kv.R || a == b || kv.lens[b] != 0) return;
    int64_t len = clamped_len(kv.lens[a], (int64_t)kv.max_pages * kv.page_tokens);
    if (keep) len = clamped_len(keep[i], len);
    const int64_t held = (len + kv.page_tokens - 1) / kv.page_tokens;
    for (int64_t j = threadIdx.x & 63; j < held; j += 64) {
        const int32_t page = kv.table[(int64_t)a * kv.max_pages + j];
        kv.table[(int64_t)b * kv.max_pages + j] = page;
        if (page >= 0 && page < kv.n_pages) atomicAdd(&kv.refs[page], 1);
    }
    if ((threadIdx.x & 63) == 0) kv.lens[b] = (int32_t)len;
}

// a wave per request: pages behind the new length are let go
__global__ __launch_bounds__(256) void truncate_kernel(KvPages kv, const int32_t *new_lens)
{
    const int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (r >= kv.R) return;
    const int T = kv.page_tokens;
    const int64_t len = clamped_len(kv.lens[r], (int64_t)kv.max_pages * T), to = clamped_len(new_lens[r], len);
    for (int64_t j = (to + T - 1) / T + (threadIdx.x & 63); j < (len + T - 1) / T; j += 64) {
        const int32_t page = kv.table[r * kv.max_pages + j];
        if (page >= 0 && page < kv.n_pages) atomicSub(&kv.refs[page], 1);
        kv.table[r * kv.max_pages + j] = -1;
    }
    if ((threadIdx.x & 63) == 0 && to != kv.lens[r]) kv.lens[r] = (int32_t)to;
}

// compact, behind count_kernel: which pages move, and where to.  list = [place that a mover goes to, by page id][holes][movers],
// pairs = [counts of the movers]
__global__ __launch_bounds__(256) void movers_kernel(KvPages kv, int32_t *scratch, int32_t *used_out)
{
    __shared__ int red[4];
    const Scratch s = carve(scratch, kv.n_pages, kv.R);
    int free_all = 0, before = 0;
    for (int b = threadIdx.x; b < s.n_blocks; b += 256) {
        free_all += s.block_free[b];
        before += b < (int)blockIdx.x ? s.block_free[b] : 0;
    }
    free_all = group_sum<256>(free_all, red);
    before = group_sum<256>(before, red);
    const int used = kv.n_pages - free_all;
    // free pages in front of place `used`: as many as there are movers
    const int edge = used / KV_COUNT_PAGES;
    int holes = 0;
    for (int b = threadIdx.x; b < edge; b += 256) holes += s.block_free[b];
    for (int64_t i = (int64_t)edge * KV_COUNT_PAGES + threadIdx.x; i < used; i += 256) holes += kv.refs[i] <= 0;
    holes = group_sum<256>(holes, red);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        s.n_pairs[0] = holes;
        *used_out = used;
    }
    constexpr int PER = KV_COUNT_PAGES / 256;
    const int64_t base = (int64_t)blockIdx.x * KV_COUNT_PAGES + threadIdx.x * PER;
    int count[PER];
    uint32_t free_bits = 0;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        count[i] = base + i < kv.n_pages ? kv.refs[base + i] : 0;
        if (base + i < kv.n_pages && count[i] <= 0) free_bits |= 1u << i;
    }
    const int free_before = before + sum_before<256>(__popc(free_bits), red);
    int32_t *place = s.list, *hole = s.list + kv.n_pages, *mover = hole + kv.n_pages;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int64_t id = base + i;
        if (id >= kv.n_pages) break;
        const int f = free_before + __popc(free_bits & ((1u << i) - 1u));   // free pages in front of id
        if (id < used) {
            if (count[i] <= 0) hole[f] = (int32_t)id;
        } else if (count[i] > 0) {
            const int k = (int)(id - f) - (used - holes);   // pages in use in front of id, less those in front of place `used`
            place[id] = k;
            mover[k] = (int32_t)id;
            s.pairs[k] = count[i];
        }
    }
}

// the same by one workgroup, without count_kernel
__global__ __launch_bounds__(1024) void movers_small_kernel(KvPages kv, int32_t *scratch, int32_t *used_out)
{
    __shared__ int red[16], prefix[SMALL_PAGES / 64];
    __shared__ u64 words[SMALL_PAGES / 64];
    const Scratch s = carve(scratch, kv.n_pages, kv.R);
    free_words(kv, words, [] {});
    __syncthreads();
    const u64 bits = (int)threadIdx.x * 64 < kv.n_pages ? words[threadIdx.x] : 0;
    const int mine = __popcll(bits);
    const int before = sum_before<1024>(mine, red), used = kv.n_pages - group_sum<1024>(mine, red);
    prefix[threadIdx.x] = before;
    const int base = threadIdx.x * 64, in_front = used <= base ? 0 : used - base >= 64 ? 64 : used - base;   // of this thread's pages, those in front of place `used`
    const int holes = group_sum<1024>(__popcll(in_front == 64 ? bits : bits & ((1ull << in_front) - 1ull)), red);
    if (threadIdx.x == 0) {
        s.n_pairs[0] = holes;
        *used_out = used;
    }
    int32_t *place = s.list, *hole = s.list + kv.n_pages, *mover = hole + kv.n_pages;
    for (int id = threadIdx.x; id < kv.n_pages; id += 1024) {
        const u64 w = words[id >> 6];
        const int f = prefix[id >> 6] + __popcll(w & ((1ull << (id & 63)) - 1ull));   // free pages in front of id
        const bool is_free = w >> (id & 63) & 1u;
        if (id < used) {
            if (is_free) hole[f] = id;
        } else if (!is_free) {
            const int k = id - f - (used - holes);
            place[id] = k;
            mover[k] = id;
            s.pairs[k] = kv.refs[id];
        }
    }
}

// tables and counts of the new order, and the copies
__global__ __launch_bounds__(256) void move_kernel(KvPages kv, int32_t *scratch, const int32_t *used_in, int32_t *table_out, int32_t *refs_out)
{
    const Scratch s = carve(scratch, kv.n_pages, kv.R);
    const int used = *used_in, moved = s.n_pairs[0];
    const int32_t *place = s.list, *hole = s.list + kv.n_pages, *mover = hole + kv.n_pages;
    const int64_t threads = (int64_t)gridDim.x * 256, me = (int64_t)blockIdx.x * 256 + threadIdx.x;
    // counts: those of pages that stay here, of holes by their rank (each element is written once)
    for (int64_t i = me; i < kv.n_pages; i += threads) {
        const int c = kv.refs[i];
        if (i >= used) refs_out[i] = 0;
        else if (c > 0) refs_out[i] = c;
    }
    for (int64_t k = me; k < moved; k += threads) refs_out[hole[k]] = s.pairs[k];
    const int64_t places = (int64_t)kv.R * kv.max_pages;
    for (int64_t i = me; i < places; i += threads) {
        const int32_t page = kv.table[i];
        int32_t to = page;
        if (page >= used && page < kv.n_pages) {
            // a page that is in a table and has no count (no state that these functions leave) stays where it is
            const int k = place[page];
            if (k >= 0 && k < moved && mover[k] == page) to = hole[k];
        }
        table_out[i] = to;
    }
    const int64_t pieces = (kv.page_bytes + COPY_PIECE - 1) / COPY_PIECE;
    for (int64_t i = blockIdx.x; i < moved * pieces; i += gridDim.x)
        copy_piece(kv.pages, kv.page_bytes, kv.n_pages, mover[i / pieces], hole[i / pieces], i % pieces);
}

}  // namespace

size_t kv_pages_scratch_words(int64_t n_pages, int64_t R)
{
    const int64_t blocks = (n_pages + KV_COUNT_PAGES - 1) / KV_COUNT_PAGES, groups = (R + KV_COUNT_REQUESTS - 1) / KV_COUNT_REQUESTS;
    return (size_t)(4 + blocks + groups + R + 3 * n_pages + (2 * R > n_pages ? 2 * R : n_pages));
}

hipError_t launch_kv_reserve(const KvPages &kv, const int32_t *grow, int32_t *granted, int32_t *scratch, hipStream_t stream)
{
    const Scratch s = carve(scratch, kv.n_pages, kv.R);
    if (kv.n_pages <= SMALL_PAGES && kv.R <= SMALL_REQUESTS) {
        reserve_small_kernel<<<1, 1024, 0, stream>>>(kv, grow, granted, scratch);
    } else {
        count_kernel<<<s.n_blocks + s.n_groups, 256, 0, stream>>>(kv, grow, scratch);
        free_kernel<<<s.n_blocks, 256, 0, stream>>>(kv, scratch);
        take_kernel<<<(kv.R + 3) / 4, 256, 0, stream>>>(kv, grow, granted, scratch);
    }
    copy_kernel<<<COPY_GROUPS, 256, 0, stream>>>(kv.pages, kv.page_bytes, kv.n_pages, s.pairs, s.pairs + 1, 2, 0, s.n_pairs);
    return hipGetLastError();
}

hipError_t launch_kv_fork(const KvPages &kv, const int32_t *src, const int32_t *dst, const int32_t *keep, int64_t n, hipStream_t stream)
{
    fork_kernel<<<(unsigned)((n + 3) / 4), 256, 0, stream>>>(kv, src, dst, keep, n);
    return hipGetLastError();
}

hipError_t launch_kv_truncate(const KvPages &kv, const int32_t *new_lens, hipStream_t stream)
{
    truncate_kernel<<<(kv.R + 3) / 4, 256, 0, stream>>>(kv, new_lens);
    return hipGetLastError();
}

hipError_t launch_kv_copy_pages(const KvPages &kv, const int32_t *src, const int32_t *dst, int64_t n, hipStream_t stream)
{
    const int64_t pieces = n * ((kv.page_bytes + COPY_PIECE - 1) / COPY_PIECE);
    copy_kernel<<<(unsigned)(pieces < COPY_GROUPS ? pieces : COPY_GROUPS), 256, 0, stream>>>(kv.pages, kv.page_bytes, kv.n_pages, src, dst, 1, n, nullptr);
    return hipGetLastError();
}

hipError_t launch_kv_compact(const KvPages &kv, int32_t *table_out, int32_t *refs_out, int32_t *used, int32_t *scratch, hipStream_t stream)
{
    const Scratch s = carve(scratch, kv.n_pages, kv.R);
    if (kv.n_pages <= SMALL_PAGES) {
        movers_small_kernel<<<1, 1024, 0, stream>>>(kv, scratch, used);
    } else {
        count_kernel<<<s.n_blocks, 256, 0, stream>>>(kv, nullptr, scratch);   // pages alone: no workgroup counts needs
        movers_kernel<<<s.n_blocks, 256, 0, stream>>>(kv, scratch, used);
    }
    move_kernel<<<COPY_GROUPS, 256, 0, stream>>>(kv, scratch, used, table_out, refs_out);
    return hipGetLastError();
}

}  // namespace ralm
