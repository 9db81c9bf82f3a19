// Kernels of the attention cache's pages (etf_kv_take, _fork, _free, _compact).  Included by etf_pages.hip, inside its anonymous namespace.
#pragma once

constexpr int PAGE_KB = 64;        // tokens of a block
constexpr int PAGE_CHUNK = 1024;   // flags of a chunk, 16 words; a multiple of it where there are very many flags
constexpr int PAGE_CHUNKS = 4096;  // most chunks

struct PageView {
    uint8_t *k, *v, *bounds;
    float *scales;
    uint16_t *tail_k, *tail_v;
    int32_t *table, *lens, *evicted;
    int32_t batch, heads, blocks, pages;
};
__device__ __forceinline__ int page_len(const PageView &c, int b) { return min(max(c.lens[b], 0), c.blocks * PAGE_KB + PAGE_KB - 1); }
__device__ __forceinline__ bool page_valid(const PageView &c, int p) { return p >= 0 && p < c.pages; }

// ------------------------------------------------------------------------------------------------
// Flags and ranks.  Which pages are free (or in use) and which blocks want a page is written down as bits, 64 to a word, with a count
// for every chunk of them; what follows works from these alone, so that nothing depends on the order in which workgroups change refs and
// table, which may be the arrays that they were read from.  The r-th page of a kind is found by a search of the chunks' sums and then
// of the chunk's words; a page's rank the other way.
// ------------------------------------------------------------------------------------------------
struct Flags {
    uint64_t *words;
    int32_t *counts;  // of each chunk
    int64_t many;     // flags
    int32_t chunks, size;  // chunks, and flags of each
};

// sum over the workgroup of 256; s_sum: four ints
__device__ __forceinline__ int group_sum(int x, int *s_sum)
{
    for (int o = 32; o; o >>= 1) x += __shfl_xor(x, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_sum[threadIdx.x >> 6] = x;
    __syncthreads();
    return s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
}

// Writes down chunk `at` of the flags flag(i), each lane its own; every thread of the workgroup calls it.
template <typename F>
__device__ __forceinline__ void put_flags(const Flags &f, int at, int *s_sum, F flag)
{
    const int64_t from = (int64_t)at * f.size;
    int sum = 0;
    for (int i0 = 0; i0 < f.size; i0 += PAGE_CHUNK) {
        bool x[PAGE_CHUNK / 256];
#pragma unroll
        for (int y = 0; y < PAGE_CHUNK / 256; ++y) {
            const int64_t i = from + i0 + 256 * y + threadIdx.x;
            x[y] = i < f.many && flag(i);
        }
#pragma unroll
        for (int y = 0; y < PAGE_CHUNK / 256; ++y) {
            const uint64_t word = __ballot(x[y]);
            if ((threadIdx.x & 63) == 0) f.words[(from + i0 + 256 * y + threadIdx.x) / 64] = word;
            sum += x[y];
        }
    }
    sum = group_sum(sum, s_sum);
    if (threadIdx.x == 0) f.counts[at] = sum;
}

// Ranks among the flags of a kind: s_upto[i] = flags set before chunk i, s_upto[chunks] = all.  Made by the whole workgroup of 256.
struct Ranks {
    const uint64_t *words;
    const int *upto;
    int chunks, size;
    int64_t many;
    __device__ __forceinline__ int all() const { return upto[chunks]; }
    // flags set before flag i
    __device__ __forceinline__ int before(int64_t i) const
    {
        const int c = (int)(i / size);
        if (c >= chunks) return all();
        int n = upto[c];
        const int64_t w0 = (int64_t)c * size / 64, w1 = i / 64;
        const uint64_t below = (1ull << (i % 64)) - 1;
        for (int64_t g = w0; g <= w1; g += 16) {
#pragma unroll
            for (int y = 0; y < 16; ++y) n += __popcll(words[g + y] & (g + y < w1 ? ~0ull : g + y == w1 ? below : 0ull));
        }
        return n;
    }
    // number of the flag with r set ones (SET) or r others before it; there is one
    template <bool SET>
    __device__ __forceinline__ int64_t find(int r) const
    {
        int lo = 0, hi = chunks - 1;  // the last chunk with no more than r before it
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            const int64_t n = SET ? (int64_t)upto[mid] : (int64_t)mid * size - upto[mid];
            if (n <= r) lo = mid;
            else hi = mid - 1;
        }
        int left = r - (int)(SET ? (int64_t)upto[lo] : (int64_t)lo * size - upto[lo]);
        const int64_t w0 = (int64_t)lo * size / 64;
        for (int g = 0; g < size / 64; g += 16) {
            uint64_t w[16];
            int sum = 0;
#pragma unroll
            for (int y = 0; y < 16; ++y) {
                w[y] = words[w0 + g + y];
                if (!SET) w[y] = ~w[y];
                sum += __popcll(w[y]);
            }
            if (left >= sum) {
                left -= sum;
                continue;
            }
            uint64_t word = 0;
            int at = 0;
            bool done = false;
#pragma unroll
            for (int y = 0; y < 16; ++y) {
                const int n = __popcll(w[y]);
                if (!done) {
                    word = w[y];
                    at = y;
                    done = left < n;
                    if (!done) left -= n;
                }
            }
            int bit = 0;  // of the word, the bit with `left` set ones below it
#pragma unroll
            for (int half = 32; half; half /= 2) {
                const int n = __popcll(word & ((1ull << half) - 1));
                if (left >= n) {
                    left -= n;
                    word >>= half;
                    bit += half;
                }
            }
            return (w0 + g + at) * 64 + bit;
        }
        return many - 1;
    }
};

// s_upto: PAGE_CHUNKS + 1 ints
__device__ __forceinline__ Ranks ranks_of(const Flags &f, int *s_upto, int *s_sum)
{
    const int per = (f.chunks + 255) / 256, from = threadIdx.x * per;
    int sum = 0;
    for (int i = from; i < min(from + per, f.chunks); ++i) {
        s_upto[i] = f.counts[i];
        sum += s_upto[i];
    }
    int x = sum;
    const int lane = threadIdx.x & 63;
    for (int o = 1; o < 64; o *= 2) {
        const int y = __shfl_up(x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();
    if (lane == 63) s_sum[threadIdx.x >> 6] = x;
    __syncthreads();
    int at = x - sum;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) at += s_sum[w];
    for (int i = from; i < min(from + per, f.chunks); ++i) {
        const int n = s_upto[i];
        s_upto[i] = at;
        at += n;
    }
    if (threadIdx.x == 255) s_upto[f.chunks] = at;
    __syncthreads();
    return Ranks{f.words, s_upto, f.chunks, f.size, f.many};
}

// ------------------------------------------------------------------------------------------------
// Take.  Slots are the blocks that an append of n tokens may complete, `per` of every (sequence, head): slot (b, h, c) is block
// lens[b] / 64 + c.  A slot that the sequence's own count completes wants a page unless it has one that no other entry names.  The
// wanting slots get the lowest free pages, in their order.
// Two launches, each a chain of dependent loads: 512 slots and 24 588 pages 3.8 and 2.3 us, 32 768 slots (22 290 of them wanting) and 438 616 pages 5.3 and
// 6.7 us (13 with 1024 slots to a workgroup).
// ------------------------------------------------------------------------------------------------
struct TakeArgs {
    PageView c;
    const int32_t *refs, *counts;
    int32_t *table_out, *refs_out, *missing;
    int n, per;
    Flags free, slots;
    int32_t *shared;  // [slots]: of a slot that wants a page, the one that others name too, or -1
};

// column of a slot, or -1 where the append does not complete that block
__device__ __forceinline__ int slot_column(const TakeArgs &a, int64_t slot, int64_t &bh)
{
    const uint32_t u = (uint32_t)slot;  // there are fewer than 2^31
    bh = u / (uint32_t)a.per;
    const int c = (int)(u % (uint32_t)a.per), b = (int)((uint32_t)bh / (uint32_t)a.c.heads), len = page_len(a.c, b);
    const int count = a.counts ? min(max(a.counts[b], 0), a.n) : a.n;
    const int64_t j = len / PAGE_KB + c;
    return j < ((int64_t)len + count) / PAGE_KB && j < a.c.blocks ? (int)j : -1;
}

__global__ __launch_bounds__(256) void k_kv_take_flags(TakeArgs a)
{
    __shared__ int s_sum[4];
    const int chunks = a.free.chunks + a.slots.chunks;
    if ((int)blockIdx.x < a.free.chunks) {
        put_flags(a.free, blockIdx.x, s_sum, [&](int64_t i) { return a.refs[i] <= 0; });
    } else if ((int)blockIdx.x < chunks) {
        put_flags(a.slots, blockIdx.x - a.free.chunks, s_sum, [&](int64_t i) {
            int64_t bh;
            const int j = slot_column(a, i, bh);
            if (j < 0) return false;
            const int p = a.c.table[bh * a.c.blocks + j], shares = page_valid(a.c, p) ? a.refs[p] : 0;
            if (shares != 1) a.shared[i] = shares > 1 ? p : -1;
            return shares != 1;
        });
    } else {  // outputs that lie elsewhere
        const int64_t at = (int64_t)(blockIdx.x - chunks) * 256 + threadIdx.x, step = (int64_t)(gridDim.x - chunks) * 256;
        if (a.refs_out != a.refs)
            for (int64_t i = at; i < a.c.pages; i += step) a.refs_out[i] = a.refs[i];
        if (a.table_out != a.c.table)
            for (int64_t i = at; i < (int64_t)a.c.batch * a.c.heads * a.c.blocks; i += step) a.table_out[i] = a.c.table[i];
    }
}

// 256 slots to a workgroup
__global__ __launch_bounds__(256) void k_kv_take(TakeArgs a)
{
    __shared__ int s_upto[PAGE_CHUNKS + 1], s_sum[4];
    const int parts = a.slots.size / 256, chunk = blockIdx.x / parts;
    const int64_t w0 = (int64_t)chunk * a.slots.size / 64, slot = (int64_t)blockIdx.x * 256 + threadIdx.x;
    int need = 0, first = 0, there = 0;  // slots that want a page: of all, before this workgroup's; free pages
    for (int i = threadIdx.x; i < a.slots.chunks; i += 256) {
        const int x = a.slots.counts[i];
        need += x;
        first += i < chunk ? x : 0;
    }
    for (int64_t w = w0 + threadIdx.x; w < (int64_t)blockIdx.x * 4; w += 256) first += __popcll(a.slots.words[w]);
    for (int i = threadIdx.x; i < a.free.chunks; i += 256) there += a.free.counts[i];
    need = group_sum(need, s_sum);
    there = group_sum(there, s_sum);
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.missing = max(0, need - there);
    if (need == 0 || need > there) return;
    first = group_sum(first, s_sum);
    const Ranks free = ranks_of(a.free, s_upto, s_sum);
    const int wave = threadIdx.x >> 6;
    uint64_t word = 0;
    for (int w = 0; w < 4; ++w) {
        const uint64_t x = a.slots.words[(int64_t)blockIdx.x * 4 + w];
        first += w < wave ? __popcll(x) : 0;
        word = w == wave ? x : word;
    }
    if (!(word >> (slot & 63) & 1)) return;
    int64_t bh;
    const int j = slot_column(a, slot, bh), shared = a.shared[slot];
    const int page = (int)free.find<true>(first + __popcll(word & ((1ull << (slot & 63)) - 1)));
    a.table_out[bh * a.c.blocks + j] = page;
    a.refs_out[page] = 1;
    if (shared >= 0) atomicSub(a.refs_out + shared, 1);
}

// ------------------------------------------------------------------------------------------------
// Compact.  With U pages in use, the i-th of the others below U takes the used page that has i used ones behind it.  All of that
// follows from the ranks, so one launch after the flags moves the pages (sources lie from U on, destinations below), and
// rewrites the table and refs.  Bound by the pages' bytes, read once and written once: 547 MB in 118 us = 4.6 TB/s (a plain copy's 5.1), 95 us = 5.8 TB/s
// where the pool was moved just before.  Pages are spread over as many workgroups as the card holds (2048) before one takes a second, 16 at a time
// at most: the ranks of 16 are found side by side.
// ------------------------------------------------------------------------------------------------
struct CompactArgs {
    PageView c;
    const int32_t *refs;
    int32_t *table_out, *refs_out, *used;
    Flags taken;
    int movers, tables;  // workgroups that move pages, that rewrite the table; the others rewrite refs
};

__global__ __launch_bounds__(256) void k_kv_used_flags(CompactArgs a)
{
    __shared__ int s_sum[4];
    put_flags(a.taken, blockIdx.x, s_sum, [&](int64_t i) { return a.refs[i] > 0; });
}

// 64 x D bytes, past the caches: 118 us where plain loads and stores take 123 (compact, 16 396 pages of 128 dimensions moved)
template <int D>
__device__ __forceinline__ void move_page(uint8_t *of, int64_t to, int64_t from, int tid)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    constexpr int PIECES = PAGE_KB * D / 16, EACH = (PIECES + 255) / 256;
    u32x4 w[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (PIECES % 256 == 0 || tid + 256 * i < PIECES) w[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(of + from * (PAGE_KB * D)) + tid + 256 * i);
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        if (PIECES % 256 == 0 || tid + 256 * i < PIECES) __builtin_nontemporal_store(w[i], reinterpret_cast<u32x4 *>(of + to * (PAGE_KB * D)) + tid + 256 * i);
}

template <int D>
__global__ __launch_bounds__(256) void k_kv_compact(CompactArgs a)
{
    constexpr int PAIRS = 16;  // pages that a workgroup moves, at most, before it looks for others
    __shared__ int s_upto[PAGE_CHUNKS + 1], s_sum[4], s_pair[PAIRS][2];
    const Ranks taken = ranks_of(a.taken, s_upto, s_sum);
    const int used = taken.all(), moving = used - taken.before(used), tid = threadIdx.x;
    if ((int)blockIdx.x < a.movers) {
        if (blockIdx.x == 0 && tid == 0) *a.used = used;
        const int each = min(PAIRS, (moving + a.movers - 1) / a.movers);
        for (int64_t i0 = (int64_t)blockIdx.x * each; i0 < moving; i0 += (int64_t)a.movers * each) {
            const int many = (int)min<int64_t>(each, moving - i0);
            __syncthreads();
            if (tid < many) s_pair[tid][0] = (int)taken.find<false>((int)(i0 + tid));
            if (tid >= 64 && tid - 64 < many) s_pair[tid - 64][1] = (int)taken.find<true>(used - 1 - (int)(i0 + tid - 64));
            __syncthreads();
            if (tid < many) {
                const int64_t to = s_pair[tid][0], from = s_pair[tid][1];
                const float2 scales = reinterpret_cast<const float2 *>(a.c.scales)[from];
                const int shares = a.refs[from];
                reinterpret_cast<float2 *>(a.c.scales)[to] = scales;
                a.refs_out[to] = shares;
                a.refs_out[from] = 0;
            }
            for (int y = 0; y < many; ++y) {
                const int64_t to = s_pair[y][0], from = s_pair[y][1];
                move_page<D>(a.c.k, to, from, tid);
                move_page<D>(a.c.v, to, from, tid);
                if (tid < 2 * D / 16) reinterpret_cast<uint4 *>(a.c.bounds + to * 2 * D)[tid] = reinterpret_cast<const uint4 *>(a.c.bounds + from * 2 * D)[tid];
            }
        }
        return;
    }
    if ((int)blockIdx.x < a.movers + a.tables) {
        const int64_t entries = (int64_t)a.c.batch * a.c.heads * a.c.blocks;
        for (int64_t i = (int64_t)(blockIdx.x - a.movers) * 256 + tid; i < entries; i += (int64_t)a.tables * 256) {
            int p = a.c.table[i];
            if (p >= used && p < a.c.pages) {
                const int before = taken.before(p);
                if (taken.words[p / 64] >> (p & 63) & 1) p = (int)taken.find<false>(used - 1 - before);
            }
            if (a.table_out != a.c.table || p != a.c.table[i]) a.table_out[i] = p;
        }
        return;
    }
    // pages that neither come nor go keep their count; what is in use no more has none
    const int64_t groups = gridDim.x - a.movers - a.tables;
    for (int64_t i = (int64_t)(blockIdx.x - a.movers - a.tables) * 256 + tid; i < a.c.pages; i += groups * 256)
        if ((taken.words[i / 64] >> (i & 63) & 1) ? i < used && a.refs_out != a.refs : i >= used) a.refs_out[i] = i < used ? a.refs[i] : 0;
}

// ------------------------------------------------------------------------------------------------
// Free: one share less of each listed page, none below zero.  3.9 us for 40 448 entries, of which 8192 are pages: a load, an atomic that returns, another.
// ------------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void k_kv_free(int32_t *refs, int pages, const int32_t *list, int64_t n)
{
    constexpr int EACH = 4;
    const int64_t from = (int64_t)blockIdx.x * 256 * EACH + threadIdx.x;
    int p[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) p[i] = from + 256 * i < n ? list[from + 256 * i] : -1;
#pragma unroll
    for (int i = 0; i < EACH; ++i)
        // whoever finds none left gives back what it took: of several at once as many find a share as there were
        if (p[i] >= 0 && p[i] < pages && atomicSub(refs + p[i], 1) <= 0) atomicAdd(refs + p[i], 1);
}

// ------------------------------------------------------------------------------------------------
// Fork.  The first launch decides what happens to every sequence and saves the rows of those sources that do not stay as they are
// themselves; the second writes every changed sequence's row, open block and lengths, and counts shares: one less for every entry that
// was there, one more for every entry that is.  32 sequences of up to 2000 tokens, 8 heads, 16 of them copied: 2.2 and 5.8 us, chains of dependent loads
// (where rows are copies already 4.3, and 5.2 with a row's table, keys and values by one workgroup).  63 copies of 187 of a sequence's 250 blocks, 8
// heads: 2.7 and 14 us, an atomic for each of 126 000 entries that go and of 94 000 that come.
// ------------------------------------------------------------------------------------------------
enum { FORK_STAYS = 0, FORK_COPY = 1, FORK_SAVED = 2, FORK_CUT = 3, FORK_EMPTY = 4 };
struct ForkArgs {
    PageView c;
    int32_t *refs;
    const int32_t *source, *keep;
    int4 *plan;         // [batch]: what happens, source, tokens, evicted
    int32_t *rows;      // saved rows of the table: [batch][heads][blocks]
    uint16_t *save_k, *save_v;  // saved open blocks: [batch][heads][64][D], [batch][heads][D][64]
    int row;            // head_dim
};

// tokens that a copy of source s made for sequence b holds: all, or as many whole blocks as keep has
__device__ __forceinline__ int fork_tokens(const ForkArgs &a, int b, int s)
{
    const int len = page_len(a.c, s);
    if (!a.keep) return len;
    const int keep = max(0, a.keep[b]);
    return keep >= len ? len : keep / PAGE_KB * PAGE_KB;
}

// The first `left` tokens of an open block's values, [D][64]: whole pieces of 8 tokens, and of the last piece only its first tokens
__device__ __forceinline__ void copy_open_values(const uint16_t *from, uint16_t *to, int row, int left)
{
    const int per = (left + 7) / 8;
    for (int i = threadIdx.x; i < row * per; i += 256) {
        const int d = i / per, p = i % per, have = min(8, left - 8 * p);
        uint4 w = reinterpret_cast<const uint4 *>(from + d * PAGE_KB)[p];
        if (have < 8) {
            const uint4 o = reinterpret_cast<const uint4 *>(to + d * PAGE_KB)[p];
            auto mix = [&](uint32_t x, uint32_t y, int at) { return have >= at + 2 ? x : have == at + 1 ? (x & 0xFFFFu) | (y & 0xFFFF0000u) : y; };
            w = make_uint4(mix(w.x, o.x, 0), mix(w.y, o.y, 2), mix(w.z, o.z, 4), mix(w.w, o.w, 6));
        }
        reinterpret_cast<uint4 *>(to + d * PAGE_KB)[p] = w;
    }
}

__global__ __launch_bounds__(256) void k_kv_fork_plan(ForkArgs a)
{
    const int64_t bh = blockIdx.x;
    const int b = (int)(bh / a.c.heads), h = (int)(bh % a.c.heads), s = a.source[b];
    int what = FORK_EMPTY, tokens = 0, evicted = 0;
    if (s >= 0 && s < a.c.batch) {
        tokens = fork_tokens(a, b, s);
        evicted = a.c.evicted[s];
        if (s == b) what = tokens == page_len(a.c, b) ? FORK_STAYS : FORK_CUT;
        else what = a.source[s] == s && fork_tokens(a, s, s) == page_len(a.c, s) ? FORK_COPY : FORK_SAVED;
    }
    if (h == 0 && threadIdx.x == 0) a.plan[b] = make_int4(what, s, tokens, evicted);
    if (what != FORK_SAVED) return;
    const int64_t from = (int64_t)s * a.c.heads + h;
    for (int j = threadIdx.x; j < tokens / PAGE_KB; j += 256) a.rows[bh * a.c.blocks + j] = a.c.table[from * a.c.blocks + j];
    const int left = tokens % PAGE_KB, D = a.row;
    if (left == 0) return;
    const int64_t tail = (from * 2 + ((tokens / PAGE_KB + evicted) & 1)) * PAGE_KB * D, save = bh * PAGE_KB * D;
    for (int i = threadIdx.x; i < left * D / 8; i += 256) reinterpret_cast<uint4 *>(a.save_k + save)[i] = reinterpret_cast<const uint4 *>(a.c.tail_k + tail)[i];
    for (int i = threadIdx.x; i < D * 8; i += 256) reinterpret_cast<uint4 *>(a.save_v + save)[i] = reinterpret_cast<const uint4 *>(a.c.tail_v + tail)[i];
}

// Three workgroups to a (sequence, head): its row of the table, its open block's keys, its values
__global__ __launch_bounds__(256) void k_kv_fork(ForkArgs a)
{
    const int64_t bh = blockIdx.x / 3;
    const int part = blockIdx.x % 3, b = (int)(bh / a.c.heads), h = (int)(bh % a.c.heads), D = a.row;
    const int4 plan = a.plan[b];
    const int what = plan.x, s = plan.y, tokens = plan.z, evicted = plan.w, full = tokens / PAGE_KB, left = tokens % PAGE_KB;
    if (what == FORK_STAYS) return;
    const int64_t from = (int64_t)s * a.c.heads + h;
    if (part == 0) {
        const int32_t *row = what == FORK_COPY ? a.c.table + from * a.c.blocks : a.rows + bh * a.c.blocks;
        int32_t *mine = a.c.table + bh * a.c.blocks;
        for (int j = threadIdx.x; j < a.c.blocks; j += 256) {
            if (what == FORK_CUT && j < full) continue;
            const int old = mine[j], now = j < full && what != FORK_EMPTY ? row[j] : -1;
            if (now == old) continue;
            if (page_valid(a.c, old)) atomicSub(a.refs + old, 1);
            if (page_valid(a.c, now)) atomicAdd(a.refs + now, 1);
            mine[j] = now;
        }
        if (h == 0 && threadIdx.x == 0) {
            a.c.lens[b] = tokens;
            a.c.evicted[b] = evicted;
        }
        return;
    }
    if (left == 0 || what == FORK_CUT) return;
    const int half = (full + evicted) & 1;
    const int64_t tail = (bh * 2 + half) * PAGE_KB * D, other = what == FORK_COPY ? (from * 2 + half) * PAGE_KB * D : bh * PAGE_KB * D;
    if (part == 2) {
        copy_open_values((what == FORK_COPY ? a.c.tail_v : a.save_v) + other, a.c.tail_v + tail, D, left);
        return;
    }
    const uint16_t *keys = (what == FORK_COPY ? a.c.tail_k : a.save_k) + other;
    for (int i = threadIdx.x; i < left * D / 8; i += 256) reinterpret_cast<uint4 *>(a.c.tail_k + tail)[i] = reinterpret_cast<const uint4 *>(keys)[i];
}
