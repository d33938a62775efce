// Pages of the shared cache among many sequences: forks that share them, pages for new
// tokens with a copy of each one that others hold too, and compaction of the pool.
//
// refs[p] counts the holders of physical page p: entries of the page table, and whatever
// else the caller keeps (a prefix that outlives its sequence).  A page with no holder is
// free; there is no list of free pages, the lowest ones are taken first, so that a call's
// result depends on its inputs alone.
//
// The tables are small beside the cache: one workgroup plans (what it needs is an order
// over all entries, a scan), and a launch of many workgroups moves the pages, which the
// memory bounds.
#include "clsa_internal.h"
#include "device_common.h"

namespace clsa {

constexpr int kPlanThreads = 1024;
constexpr int kForkEntries = kMaxForkBatch;  // table entries of a fork's workgroup (64 KB of LDS)
constexpr int kCopyBytes = 8192;       // a copying workgroup's piece of a page
// Copies of this many bytes go past the caches.
constexpr int64_t kCopyStreamed = (int64_t)64 << 20;

struct PageArgs {
    int32_t *table, *refs;
    int batch, max_pages, pages;
};

// ---- fork ----

struct ForkArgs : PageArgs {
    const int32_t *parent;
    int32_t *seq_lens;
    int cols;
};

// One workgroup = `cols` columns of the table, whole; the last one takes the lengths.
// Every entry is read before one is written, so that a slot may take from one that
// changes in the same call.
__global__ __launch_bounds__(256) void pages_fork_kernel(ForkArgs a) {
    __shared__ int32_t s_old[kForkEntries];
    if (blockIdx.x == gridDim.x - 1) {
        for (int b = threadIdx.x; b < a.batch; b += 256) s_old[b] = a.seq_lens[b];
        __syncthreads();
        for (int b = threadIdx.x; b < a.batch; b += 256) {
            const int up = a.parent[b];
            if (up < -1 || up >= a.batch) note_device_error(kDevErrPages);  // stays as it is
            else if (up != b) a.seq_lens[b] = up < 0 ? 0 : s_old[up];
        }
        return;
    }
    const int c0 = blockIdx.x * a.cols, width = min(a.cols, a.max_pages - c0), n = a.batch * width;
    int32_t *table = a.table + c0;
    for (int i0 = threadIdx.x; i0 < n; i0 += 1024) {  // four loads in flight
        int v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + 256 * j, b = i / width;
            if (i < n) v[j] = table[(size_t)b * a.max_pages + (i - b * width)];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i0 + 256 * j < n) s_old[i0 + 256 * j] = v[j];
    }
    __syncthreads();
    for (int i0 = threadIdx.x; i0 < n; i0 += 1024) {
        int up[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + 256 * j;
            up[j] = i < n ? a.parent[i / width] : -2;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int i = i0 + 256 * j, b = i / width, c = i - b * width;
            if (up[j] < -1 || up[j] >= a.batch || up[j] == b) continue;
            const int old = s_old[i], from = up[j] < 0 ? -1 : s_old[up[j] * width + c];
            const bool held = from >= 0 && from < a.pages;
            if (from < -1 || from >= a.pages || old < -1 || old >= a.pages) note_device_error(kDevErrPages);
            const int now = held ? from : -1;
            if (now == old) continue;
            table[(size_t)b * a.max_pages + c] = now;
            if (held) atomicAdd(a.refs + now, 1);
            if (old >= 0 && old < a.pages) atomicSub(a.refs + old, 1);
        }
    }
}

hipError_t launch_pages_fork(const Geometry &g, int pages, const int32_t *parent, int32_t *table,
                             int32_t *seq_lens, int32_t *refs, hipStream_t stream) {
    if (g.batch > kForkEntries) return hipErrorInvalidValue;
    // about 1024 entries a workgroup, whole 16-byte pieces of a row where that many fit
    // (72 slots x 235 pages: 64 columns 13.1 us, 12 3.9)
    ForkArgs a{{table, refs, g.batch, g.max_pages, pages}, parent, seq_lens, 1024 / g.batch / 4 * 4};
    a.cols = a.cols < 4 ? (4 * g.batch <= kForkEntries ? 4 : kForkEntries / g.batch) : a.cols < 64 ? a.cols : 64;
    pages_fork_kernel<<<dim3(div_up(g.max_pages, a.cols) + 1), dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

// ---- moving pages ----

// Pairs of pages (source, destination), their number known on the device; a pair without
// a source (-1) is skipped.  A page is cut into pieces over all of its tensors.
struct CopyArgs {
    char *data[kMaxPaged];
    int64_t bytes[kMaxPaged];   // of a page
    int first[kMaxPaged + 1];   // piece numbers
    int tensors, pages;
    int64_t page_bytes;         // of all tensors
    const int32_t *src, *dst, *count;  // count: null if n is known
    int n;
    unsigned grid, step_pairs, step_pieces;  // copying workgroups, and their number in pairs and pieces
};

// One piece: N 16-byte loads a thread in flight.  NT: streamed past the caches.
template <bool NT>
__device__ __forceinline__ void copy_piece(const char *from, char *to, int len) {
    constexpr int N = kCopyBytes / 16 / 256;
    u32x4 v[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int o = (threadIdx.x + 256 * j) * 16;
        const u32x4 *p = reinterpret_cast<const u32x4 *>(from + o);
        if (o < len) v[j] = NT ? __builtin_nontemporal_load(p) : *p;
    }
#pragma unroll
    for (int j = 0; j < N; ++j) {
        const int o = (threadIdx.x + 256 * j) * 16;
        u32x4 *p = reinterpret_cast<u32x4 *>(to + o);
        if (o < len) {
            if (NT) __builtin_nontemporal_store(v[j], p);
            else *p = v[j];
        }
    }
}

// Work item i: piece i % per of pair i / per.  The pairs' lists have room for every item of
// the launch, so that a pair is loaded along with their number.
__device__ __forceinline__ void copy_pages(const CopyArgs &a) {
    const int per = a.first[a.tensors];
    uint32_t k = blockIdx.x / (uint32_t)per, piece = blockIdx.x - k * per;
    int src = a.src[k], dst = a.dst[k];
    const int n = a.count ? *a.count : a.n;
    const bool stream = (int64_t)n * a.page_bytes >= kCopyStreamed;
    while (k < (uint32_t)n) {
        if (src != -1 && src != dst) {
            if (src < 0 || src >= a.pages || dst < 0 || dst >= a.pages) {
                if (piece == 0 && threadIdx.x == 0) note_device_error(kDevErrPages);
            } else {
                int t = 0;
                while ((int)piece >= a.first[t + 1]) ++t;
                const int64_t bytes = a.bytes[t], at = (int64_t)((int)piece - a.first[t]) * kCopyBytes;
                const int len = (int)min((int64_t)kCopyBytes, bytes - at);
                const char *from = a.data[t] + src * bytes + at;
                char *to = a.data[t] + dst * bytes + at;
                if (((uintptr_t)a.data[t] | bytes) % 16 != 0) {
                    for (int o = threadIdx.x * 4; o < len; o += 1024)
                        *reinterpret_cast<uint32_t *>(to + o) = *reinterpret_cast<const uint32_t *>(from + o);
                } else if (stream) {
                    copy_piece<true>(from, to, len);
                } else {
                    copy_piece<false>(from, to, len);
                }
            }
        }
        k += a.step_pairs;
        piece += a.step_pieces;
        if (piece >= (uint32_t)per) {
            piece -= per;
            ++k;
        }
        if (k >= (uint32_t)n) break;
        src = a.src[k];
        dst = a.dst[k];
    }
}

__global__ __launch_bounds__(256) void pages_copy_kernel(CopyArgs a) {
    copy_pages(a);
}

// For at most n pairs, whose lists have that many places.
static void copy_args(CopyArgs &a, int pages, int tensors, const PagedTensor *t, int64_t n) {
    a.pages = pages;
    a.tensors = tensors;
    int per = 0;
    for (int i = 0; i < tensors; ++i) {
        a.data[i] = static_cast<char *>(t[i].data);
        a.bytes[i] = t[i].page_bytes;
        a.page_bytes += t[i].page_bytes;
        a.first[i] = per;
        per += (int)((t[i].page_bytes + kCopyBytes - 1) / kCopyBytes);
    }
    a.first[tensors] = per;
    // a workgroup for each piece, eight a CU at most: those that find no pair cost their launch
    a.grid = (unsigned)(n * per < 2048 ? n * per : 2048);
    if (per) {
        a.step_pairs = a.grid / per;
        a.step_pieces = a.grid % per;
    }
}

hipError_t launch_pages_copy(int pages, int tensors, const PagedTensor *t, int n,
                             const int32_t *src, const int32_t *dst, hipStream_t stream) {
    if (n == 0 || tensors == 0) return hipSuccess;
    CopyArgs a{};
    copy_args(a, pages, tensors, t, n);
    a.src = src;
    a.dst = dst;
    a.n = n;
    pages_copy_kernel<<<dim3(a.grid), dim3(256), 0, stream>>>(a);
    return hipGetLastError();
}

// ---- reserve ----

// Sum of v over the threads before this one, and over all of them (T threads).
template <int T>
__device__ __forceinline__ int block_scan(int v, int *s, int &all) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const int y = __shfl_up(x, m);
        if (lane >= m) x += y;
    }
    if (lane == 63) s[wave] = x;
    __syncthreads();
    int before = 0;
    all = 0;
#pragma unroll
    for (int w = 0; w < T / 64; ++w) {
        if (w < wave) before += s[w];
        all += s[w];
    }
    __syncthreads();
    return before + x - v;
}

// refs are counted by atomics and read past the first-level cache.
__device__ __forceinline__ int ref_of(const int32_t *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

struct ReserveArgs {
    PageArgs p;
    const int32_t *start, *count;
    int32_t *missing;
    int32_t *state, *src, *dst, *n_pairs;  // workspace: [entries] each, and one number
    int n_q, max_len, page_shift, slots;
};

// The table entry of (sequence, slot) i, where its new tokens reach it: the page index.
__device__ __forceinline__ bool reserve_entry(const ReserveArgs &a, int i, size_t &at) {
    const int b = i / a.slots, slot = i - b * a.slots;
    const int first = a.start[b], n = min(max(a.count[b], 0), a.n_q);
    if (first < 0 || first > a.max_len) return false;
    const int end = first + min(n, a.max_len - first), page = (first >> a.page_shift) + slot;
    at = (size_t)b * a.p.max_pages + page;
    return first < end && (int64_t)page << a.page_shift < end;
}

// One workgroup.  An entry without a page needs one; so does an entry whose page others
// hold and that do not all write now: it gets a copy.  Where every holder of a page
// writes, the last of them (by sequence) keeps it.  To find out, each writer drops its
// count; a count of zero says that all holders write, and the counter itself then takes
// the largest entry number, as the least negative value below zero.
__global__ __launch_bounds__(kPlanThreads) void pages_reserve_kernel(ReserveArgs a) {
    __shared__ int s_scan[kPlanThreads / 64];
    const int tid = threadIdx.x, entries = a.p.batch * a.slots;
    int32_t *refs = a.p.refs;
    __shared__ uint32_t s_odd;
    if (tid == 0) s_odd = 0u;
    __syncthreads();
    uint32_t odd = 0u;  // what the entries and ranges hold that they should not
    for (int b = tid; b < a.p.batch; b += kPlanThreads) {
        const int first = a.start[b], n = a.count[b];
        if (first < 0 || first > a.max_len || n < 0 || n > a.n_q || n > a.max_len - first) odd |= kDevErrAppend;
    }
    constexpr int kNone = -2, kNew = -1;  // state: not reached, has no page; else its page
    for (int i = tid; i < entries; i += kPlanThreads) {
        size_t at;
        int st = kNone;
        if (reserve_entry(a, i, at)) {
            st = a.p.table[at];
            if (st < 0 || st >= a.p.pages) {
                if (st != -1) odd |= kDevErrPages;
                st = kNew;
            } else {
                atomicSub(refs + st, 1);
            }
        }
        a.state[i] = st;
    }
    if (odd) atomicOr(&s_odd, odd);
    __threadfence();
    __syncthreads();
    for (int i = tid; i < entries; i += kPlanThreads) {
        const int st = a.state[i];
        if (st >= 0 && ref_of(refs + st) <= 0) atomicMin(refs + st, -(i + 1));
    }
    __threadfence();
    __syncthreads();
    // needs in the order of entries; a keeper leaves the list once everyone has looked
    int need = 0;
    for (int i0 = 0; i0 < entries; i0 += kPlanThreads) {
        const int i = i0 + tid;
        const int st = i < entries ? a.state[i] : kNone;
        const bool keeps = st >= 0 && ref_of(refs + st) == -(i + 1);
        const bool wants = st != kNone && !keeps;
        int all;
        const int k = need + block_scan<kPlanThreads>(wants, s_scan, all);
        if (wants) {
            a.src[k] = st;   // -1: nothing to copy
            a.dst[k] = i;    // the entry, until its page is known
        }
        if (keeps) a.state[i] = -3 - st;
        need += all;
    }
    __threadfence();
    __syncthreads();
    for (int i = tid; i < entries; i += kPlanThreads)
        if (a.state[i] <= -3) __hip_atomic_store(refs + (-3 - a.state[i]), 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __threadfence();
    __syncthreads();
    // the lowest free pages, as many as are needed (state holds them from here on)
    int found = 0;
    for (int p0 = 0; p0 < a.p.pages && found < need; p0 += 4 * kPlanThreads) {
        const int p = p0 + 4 * tid;
        int free[4], n = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            free[j] = p + j < a.p.pages && ref_of(refs + p + j) == 0;
            n += free[j];
        }
        int all;
        int k = found + block_scan<kPlanThreads>(n, s_scan, all);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if (free[j] && k < need) a.state[k] = p + j;
            k += free[j];
        }
        found += all;
    }
    __threadfence();
    __syncthreads();
    const bool enough = found >= need;
    for (int k = tid; k < need; k += kPlanThreads) {
        const int src = a.src[k];
        if (enough) {
            size_t at;
            reserve_entry(a, a.dst[k], at);
            const int page = a.state[k];
            a.p.table[at] = page;
            refs[page] = 1;
            a.dst[k] = page;
        } else if (src >= 0) {
            atomicAdd(refs + src, 1);  // nothing happens: its holder holds it still
        }
    }
    if (tid == 0) {
        *a.n_pairs = enough ? need : 0;
        *a.missing = enough ? 0 : need - found;
        const uint32_t bits = s_odd | (enough ? 0u : kDevErrPages);
        if (bits) note_device_error(bits);
    }
}

// The same for at most T entries, one a thread.  A page that is free stays free until it is
// taken, so the first free ones are looked up while the entries are on their way, and the
// writers of a page that others hold meet in a hash table in LDS: no counter changes
// before the call is known to have enough pages.
template <int T>
__global__ __launch_bounds__(T) void pages_reserve_few_kernel(ReserveArgs a) {
    constexpr int H = 2 * T, N = 2048 / T;  // hash slots; pages a thread looks at in a turn
    __shared__ int s_scan[T / 64], s_key[H], s_writers[H], s_last[H], s_free[T];
    __shared__ uint32_t s_odd;
    const int tid = threadIdx.x;
    int32_t *refs = a.p.refs;
    // the entry's chain of loads first (range, table, holders), the first pages' refs beside it
    uint32_t odd = 0u;
    size_t at = 0;
    const bool reached = tid < a.p.batch * a.slots && reserve_entry(a, tid, at);
    bool free[N];
#pragma unroll
    for (int j = 0; j < N; ++j) free[j] = N * tid + j < a.p.pages && refs[N * tid + j] == 0;
    int src = -1, held = 0, h = 0;
    if (reached) {
        src = a.p.table[at];
        if (src < -1 || src >= a.p.pages) odd |= kDevErrPages;
        if (src < 0 || src >= a.p.pages) src = -1;
        else held = refs[src];
    }
    for (int b = tid; b < a.p.batch; b += T) {
        const int first = a.start[b], n = a.count[b];
        if (first < 0 || first > a.max_len || n < 0 || n > a.n_q || n > a.max_len - first) odd |= kDevErrAppend;
    }
    if (tid == 0) s_odd = 0u;
    for (int h = tid; h < H; h += T) {
        s_key[h] = -1;
        s_writers[h] = 0;
        s_last[h] = -1;
    }
    __syncthreads();
    if (reached) {
        if (src >= 0 && held != 1) {
            h = (int)(((uint32_t)src * 2654435761u) >> 16) & (H - 1);
            for (;;) {  // at most T keys in 2 T slots
                const int key = atomicCAS(&s_key[h], -1, src);
                if (key == -1 || key == src) break;
                h = (h + 1) & (H - 1);
            }
            atomicAdd(&s_writers[h], 1);
            atomicMax(&s_last[h], tid);
        }
    }
    if (odd) atomicOr(&s_odd, odd);
    __syncthreads();
    const bool keeps = src >= 0 && (held == 1 || (s_writers[h] == held && s_last[h] == tid));
    const bool wants = reached && !keeps;
    int need;
    const int k = block_scan<T>(wants, s_scan, need);
    int found = 0;
    for (int p0 = 0; found < need;) {
        int n = 0, all;
#pragma unroll
        for (int j = 0; j < N; ++j) n += free[j];
        int f = found + block_scan<T>(n, s_scan, all);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (free[j] && f < need) s_free[f] = p0 + N * tid + j;
            f += free[j];
        }
        found += all;
        p0 += N * T;
        if (p0 >= a.p.pages) break;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int p = p0 + N * tid + j;
            free[j] = p < a.p.pages && refs[p] == 0;
        }
    }
    __syncthreads();
    const bool enough = found >= need;
    if (wants && enough) {
        const int page = s_free[k];
        a.p.table[at] = page;
        refs[page] = 1;
        a.src[k] = src;  // -1: nothing to copy
        a.dst[k] = page;
        if (src >= 0) atomicSub(refs + src, 1);
    }
    if (tid == 0) {
        *a.n_pairs = enough ? need : 0;
        *a.missing = enough ? 0 : need - found;
        const uint32_t bits = s_odd | (enough ? 0u : kDevErrPages);
        if (bits) note_device_error(bits);
    }
}

static int reserve_slots(const Geometry &g) {
    return (int)(((int64_t)g.n_q + (1 << g.page_shift) - 2) / (1 << g.page_shift) + 1);
}

size_t reserve_ws_ints(const Geometry &g) {
    return (size_t)g.batch * reserve_slots(g) * 3 + 64;
}

bool reserve_supported(const Geometry &g) { return (int64_t)g.batch * reserve_slots(g) < (1 << 24); }

hipError_t launch_pages_reserve(const Geometry &g, int pages, int tensors, const PagedTensor *t,
                                const int32_t *start, const int32_t *count, int32_t *table,
                                int32_t *refs, int32_t *missing, int32_t *ws, hipStream_t stream) {
    if (!reserve_supported(g)) return hipErrorInvalidValue;
    ReserveArgs a;
    a.p = {table, refs, g.batch, g.max_pages, pages};
    a.start = start;
    a.count = count;
    a.missing = missing;
    a.n_q = g.n_q;
    a.max_len = g.max_len;
    a.page_shift = g.page_shift;
    a.slots = reserve_slots(g);
    const size_t entries = (size_t)g.batch * a.slots;
    a.n_pairs = ws;
    a.state = ws + 64;
    a.src = a.state + entries;
    a.dst = a.src + entries;
    if (entries <= 256) pages_reserve_few_kernel<256><<<dim3(1), dim3(256), 0, stream>>>(a);
    else if (entries <= kPlanThreads) pages_reserve_few_kernel<kPlanThreads><<<dim3(1), dim3(kPlanThreads), 0, stream>>>(a);
    else pages_reserve_kernel<<<dim3(1), dim3(kPlanThreads), 0, stream>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || tensors == 0) return e;
    CopyArgs c{};
    copy_args(c, pages, tensors, t, (int64_t)entries);
    c.src = a.src;
    c.dst = a.dst;
    c.count = a.n_pairs;
    pages_copy_kernel<<<dim3(c.grid), dim3(256), 0, stream>>>(c);
    return hipGetLastError();
}

// ---- compact ----

struct CompactArgs {
    PageArgs p;
    int32_t *bound;
    int32_t *held, *to, *src, *dst, *n_pairs;  // workspace: [pages] each, and one number
};

// Table entries that hold each page (held: zero on entry).
__global__ __launch_bounds__(256) void pages_count_kernel(CompactArgs a) {
    const size_t n = (size_t)a.p.batch * a.p.max_pages;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
        const int e = a.p.table[i];
        if (e >= 0 && e < a.p.pages) atomicAdd(a.held + e, 1);
        else if (e != -1) note_device_error(kDevErrPages);
    }
}

// Pools whose pages one workgroup counts in LDS, and the tables that it goes through itself.
constexpr int kLdsPages = 8192;
constexpr int kLdsEntries = 32768;

// One workgroup: with U pages in use, the k-th page from U on that the table alone holds
// moves to the k-th free page below U.  There are at least as many of those; a page that
// something else holds stays.  COUNT: it makes the table's counts as well, in LDS.
template <bool COUNT>
__global__ __launch_bounds__(kPlanThreads) void pages_compact_kernel(CompactArgs a) {
    constexpr int N = 8;  // consecutive pages a thread looks at in a turn
    __shared__ int s_scan[kPlanThreads / 64];
    __shared__ int s_bound, s_odd;
    __shared__ int32_t s_held[COUNT ? kLdsPages : 1];
    __shared__ uint16_t s_src[COUNT ? kLdsPages / 2 : 1], s_dst[COUNT ? kLdsPages : 1];
    const int tid = threadIdx.x;
    int r[N], mine = 0;
    if (COUNT)
        for (int p = tid; p < a.p.pages; p += kPlanThreads) s_held[p] = 0;
    if (tid == 0) s_bound = s_odd = 0;
    for (int p0 = 0; p0 < a.p.pages; p0 += N * kPlanThreads)
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int p = p0 + N * tid + j;
            r[j] = p < a.p.pages ? a.p.refs[p] : 0;
            mine += r[j] > 0;
        }
    int used;
    block_scan<kPlanThreads>(mine, s_scan, used);
    if (COUNT) {
        bool odd = false;
        const int n = a.p.batch * a.p.max_pages;
        for (int i0 = 0; i0 < n; i0 += 4 * kPlanThreads) {
            int e[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int i = i0 + j * kPlanThreads + tid;
                e[j] = i < n ? a.p.table[i] : -1;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (e[j] >= 0 && e[j] < a.p.pages) atomicAdd(&s_held[e[j]], 1);
                else odd |= e[j] != -1;
            }
        }
        if (odd) s_odd = 1;
        __syncthreads();
    }
    int holes = 0, moves = 0, bound = 0;
    for (int p0 = 0; p0 < a.p.pages; p0 += N * kPlanThreads) {
        const int first = p0 + N * tid;
        int n = 0;  // holes, and moves in the high half
        bool hole[N], move[N];
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int p = first + j;
            const bool in = p < a.p.pages;
            if (a.p.pages > N * kPlanThreads) r[j] = in ? a.p.refs[p] : 0;
            hole[j] = in && p < used && r[j] <= 0;
            move[j] = in && p >= used && r[j] > 0 && r[j] == (COUNT ? s_held[p] : a.held[p]);
            n += hole[j] + (move[j] << 16);
            if (in) a.to[p] = p;
            if (r[j] > 0 && !move[j]) bound = p + 1;
        }
        int all;
        const int before = block_scan<kPlanThreads>(n, s_scan, all);
        int h = holes + (before & 0xffff), m = moves + (before >> 16);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            if (COUNT) {
                if (hole[j]) s_dst[h++] = (uint16_t)(first + j);
                if (move[j]) s_src[m++] = (uint16_t)(first + j);
            } else {
                if (hole[j]) a.dst[h++] = first + j;
                if (move[j]) a.src[m++] = first + j;
            }
        }
        holes += all & 0xffff;
        moves += all >> 16;
    }
    if (bound) atomicMax(&s_bound, bound);
    __threadfence_block();
    __syncthreads();
    for (int k = tid; k < moves; k += kPlanThreads) {
        const int src = COUNT ? s_src[k] : a.src[k], dst = COUNT ? s_dst[k] : a.dst[k];
        if (COUNT) {
            a.src[k] = src;
            a.dst[k] = dst;
        }
        a.to[src] = dst;
        a.p.refs[dst] = COUNT ? s_held[src] : a.held[src];  // all of its holders are entries
        a.p.refs[src] = 0;
    }
    if (tid == 0) {
        *a.n_pairs = moves;
        *a.bound = max(s_bound, moves ? (COUNT ? s_dst[moves - 1] : a.dst[moves - 1]) + 1 : 0);
        if (s_odd) note_device_error(kDevErrPages);
    }
}

struct MoveArgs {
    CompactArgs a;
    CopyArgs c;
};

__global__ __launch_bounds__(256) void pages_move_kernel(MoveArgs m) {
    const CompactArgs &a = m.a;
    const size_t n = (size_t)a.p.batch * a.p.max_pages;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) {
        const int e = a.p.table[i];
        if (e >= 0 && e < a.p.pages) {
            const int now = a.to[e];
            if (now != e) a.p.table[i] = now;
        }
    }
    if (m.c.tensors && blockIdx.x < m.c.grid) copy_pages(m.c);
}

size_t compact_ws_ints(int pages) { return (size_t)pages * 4 + 64; }

hipError_t launch_pages_compact(const Geometry &g, int pages, int tensors, const PagedTensor *t,
                                int32_t *table, int32_t *refs, int32_t *bound, int32_t *ws,
                                hipStream_t stream) {
    CompactArgs a;
    a.p = {table, refs, g.batch, g.max_pages, pages};
    a.bound = bound;
    a.n_pairs = ws;
    a.held = ws + 64;
    a.to = a.held + pages;
    a.src = a.to + pages;
    a.dst = a.src + pages;
    const size_t n = (size_t)g.batch * g.max_pages;
    const unsigned grid = (unsigned)(n < 2048 * 256 ? (n + 255) / 256 : 2048);
    if (pages <= kLdsPages && n <= kLdsEntries) {
        pages_compact_kernel<true><<<dim3(1), dim3(kPlanThreads), 0, stream>>>(a);
    } else {
        hipError_t e = launch_zero_u32(reinterpret_cast<uint32_t *>(a.held), (size_t)pages, stream);
        if (e != hipSuccess) return e;
        pages_count_kernel<<<dim3(grid), dim3(256), 0, stream>>>(a);
        pages_compact_kernel<false><<<dim3(1), dim3(kPlanThreads), 0, stream>>>(a);
    }
    MoveArgs m{a, {}};
    // at most half of the pages move, and at least one pair has room
    if (tensors) copy_args(m.c, pages, tensors, t, (pages + 1) / 2);
    m.c.src = a.src;
    m.c.dst = a.dst;
    m.c.count = a.n_pairs;
    pages_move_kernel<<<dim3(grid > m.c.grid ? grid : m.c.grid), dim3(256), 0, stream>>>(m);
    return hipGetLastError();
}

hipError_t take_device_error_pages(uint32_t *bits) { return take_source_device_error(bits); }

}  // namespace clsa
