// Rows of the vocabulary table for a rank's slots, and the table's gradient by sorted tokens (wlb_embed_fwd / wlb_embed_bwd).
#include <algorithm>
#include <cmath>

#include "wlb_device.h"
#include "wlb_vocab.h"

namespace wlb {

wlb_status check_vocab(const wlb_vocab_desc* d, const char* call, int32_t allowed) {
    if (!d) return fail(WLB_ERR_INVALID_ARG, "%s: null desc", call);
    if (d->n_q < 1 || d->t_kv < 1 || d->n_docs < 1 || d->vocab < 1 || d->hidden < 1)
        return fail(WLB_ERR_INVALID_ARG, "%s: n_q=%d t_kv=%d n_docs=%d vocab=%d hidden=%d", call, d->n_q, d->t_kv, d->n_docs, d->vocab, d->hidden);
    if (!(d->scale > 0.0f) || !std::isfinite(d->scale)) return fail(WLB_ERR_INVALID_ARG, "%s: scale must be finite and > 0", call);
    if (d->flags & ~allowed) return fail(WLB_ERR_INVALID_ARG, "%s: flags 0x%x (0x%x apply)", call, d->flags, allowed);
    if (d->hidden % 8 != 0 || d->hidden > 65536) return fail(WLB_ERR_UNSUPPORTED, "%s: hidden=%d (a multiple of 8 up to 65536)", call, d->hidden);
    if (d->vocab > (1 << 30) || d->n_q > (1 << 30)) return fail(WLB_ERR_UNSUPPORTED, "%s: vocab=%d or n_q=%d above 2^30", call, d->vocab, d->n_q);
    return WLB_OK;
}

// The word that slot i holds, `none` for padding and for tokens that are no word.
__device__ __forceinline__ int slot_word(const int32_t* tokens, const int32_t* q_idx, int i, int t_kv, int vocab, int none) {
    const int g = q_idx[i];
    if ((unsigned)g >= (unsigned)t_kv) return none;
    const int w = tokens[g];
    return (unsigned)w < (unsigned)vocab ? w : none;
}

__device__ __forceinline__ float bf16_to_f32(uint32_t bits16) { return __builtin_bit_cast(float, bits16 << 16); }

// two bf16 in a register <-> floats
__device__ __forceinline__ void unpack2(uint32_t p, float& a, float& b) { a = bf16_to_f32(p & 0xffffu); b = __builtin_bit_cast(float, p & 0xffff0000u); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    bf16x2 r;
    r[0] = (__bf16)a; r[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, r);
}

// ------------------------------------------------------------------------------------------
// Lookup.  Nothing but copies: bound by memory.  A row is taken by `lanes` threads (a power of two, 16 bytes each a step), and a
// thread has kLookupRows rows under way, since a row's load waits for its token and the token for its slot.
constexpr int kLookupRows = 4;

__global__ void __launch_bounds__(256) embed_fwd_kernel(const int32_t* tokens, const int32_t* q_idx, const uint4* table, uint4* x, int n_q, int t_kv, int vocab,
                                                        int chunks, int lanes_log2, float scale) {
    const int lanes = 1 << lanes_log2, per_pass = 256 >> lanes_log2;
    const int row0 = (int)blockIdx.x * (per_pass * kLookupRows) + ((int)threadIdx.x >> lanes_log2), lane = threadIdx.x & (lanes - 1);
    int word[kLookupRows];
#pragma unroll
    for (int r = 0; r < kLookupRows; ++r) {
        const int i = row0 + r * per_pass;
        word[r] = i < n_q ? slot_word(tokens, q_idx, i, t_kv, vocab, -1) : -1;
    }
    for (int c = lane; c < chunks; c += lanes) {
        uint4 v[kLookupRows];
#pragma unroll
        for (int r = 0; r < kLookupRows; ++r) v[r] = word[r] >= 0 ? table[(size_t)word[r] * chunks + c] : uint4{0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < kLookupRows; ++r) {
            const int i = row0 + r * per_pass;
            if (i >= n_q) continue;
            uint32_t p[4] = {v[r].x, v[r].y, v[r].z, v[r].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float a, b;
                unpack2(p[k], a, b);
                p[k] = pack2(scale * a, scale * b);
            }
            // a row that is not looked up is 0 whatever the scale
            x[(size_t)i * chunks + c] = word[r] >= 0 ? uint4{p[0], p[1], p[2], p[3]} : uint4{0, 0, 0, 0};
        }
    }
}

// ------------------------------------------------------------------------------------------
// Sort of the slots by word, stable: slots of one word stay in order and the sums over them are reproducible.  Slots without a word get
// the key `vocab` and end up last.
//
// Up to kSearchMost slots: a slot's place is the number of slots that come before it.  Tiles of 256 slots are sorted by comparing all with
// all, then every slot finds its place among each tile's words by a binary search, on the whole GPU (16408 slots: 18 us in all; one workgroup sorting by
// digits took 38 us for half as many).  The searches grow with the square of the slots.  Above that digit by digit, three launches a pass.  The whole gradient at
// hidden 64, by search and by digits, us: 16384 slots, 32768 words 29 and 45 (131072 words: 33 and 52), 32768 slots 36 and 49 (42 and 58), 49152 slots 51 and 54 (58
// and 64), 65536 slots 70 and 59 (72 and 68), 131072 slots 192 and 76 (194 and 92).
// Up to kDirectMost slots: one launch, in which workgroups of kDirectSlots slots compare them with all (372 slots: 5 us, the three launches 9).
constexpr int kDirectMost = 1024, kDirectSlots = 64;
constexpr int kSearchMost = 53248, kSearchTile = 256, kSearchGroup = 16;       // tiles that a workgroup searches
constexpr int kSortThreads = 1024, kSortWaves = kSortThreads / 64, kDigitBits = 9;
constexpr int kSortBlock = 4 * kSortThreads;                    // slots per workgroup of the sort by digits

struct SortArgs {
    const int32_t *tokens, *q_idx;
    int32_t *word[2], *slot[2];     // the sorted list ends up in [0]; [1]: ping-pong, or words by tile, sorted, and slots' places in their tile
    uint32_t* hist;                 // by digits: [bins][blocks] of a pass; by search: [blocks][n_q] slots of a group of tiles that come before
    int n_q, t_kv, vocab, passes, bits, blocks;
};

// Sixteen threads to a slot, each compares it with a sixteenth of all.
__global__ void __launch_bounds__(kDirectMost) sort_direct_kernel(SortArgs a) {
    constexpr int W = kDirectMost / kDirectSlots, J = kDirectMost / W;
    __shared__ __attribute__((aligned(16))) int s_key[kDirectMost];
    __shared__ int s_count[W][kDirectSlots];
    const int tid = threadIdx.x, x = tid % kDirectSlots, y = tid / kDirectSlots, i = (int)blockIdx.x * kDirectSlots + x;
    s_key[tid] = tid < a.n_q ? slot_word(a.tokens, a.q_idx, tid, a.t_kv, a.vocab, a.vocab) : 0x7ffffffe;
    __syncthreads();
    const int key = s_key[i];
    // j comes before i: its word is smaller, or the same and j < i
    int count = 0;
#pragma unroll
    for (int j = 0; j < J; j += 4) {
        const int4 other = *reinterpret_cast<const int4*>(s_key + y * J + j);
        const int ahead = i - (y * J + j);
        count += (other.x < key + (ahead > 0)) + (other.y < key + (ahead > 1)) + (other.z < key + (ahead > 2)) + (other.w < key + (ahead > 3));
    }
    s_count[y][x] = count;
    __syncthreads();
    if (y > 0 || i >= a.n_q) return;
#pragma unroll
    for (int w = 1; w < W; ++w) count += s_count[w][x];
    a.word[0][count] = key;
    a.slot[0][count] = i;
}

// Four threads to a slot, each compares it with a quarter of its tile.
__global__ void __launch_bounds__(4 * kSearchTile) sort_tile_kernel(SortArgs a) {
    __shared__ __attribute__((aligned(16))) int s_key[kSearchTile];
    __shared__ int s_count[3][kSearchTile];
    const int tid = threadIdx.x % kSearchTile, quarter = threadIdx.x / kSearchTile, i = (int)blockIdx.x * kSearchTile + tid;
    if (quarter == 0) s_key[tid] = i < a.n_q ? slot_word(a.tokens, a.q_idx, i, a.t_kv, a.vocab, a.vocab) : 0x7ffffffe;
    __syncthreads();
    const int key = s_key[tid], j0 = quarter * (kSearchTile / 4);
    // j comes before i: its word is smaller, or the same and j < i
    int count = 0;
#pragma unroll
    for (int j = 0; j < kSearchTile / 4; j += 4) {
        const int4 other = *reinterpret_cast<const int4*>(s_key + j0 + j);
        const int ahead = tid - (j0 + j);
        count += (other.x < key + (ahead > 0)) + (other.y < key + (ahead > 1)) + (other.z < key + (ahead > 2)) + (other.w < key + (ahead > 3));
    }
    if (quarter > 0) s_count[quarter - 1][tid] = count;
    __syncthreads();
    if (quarter > 0) return;
    count += s_count[0][tid] + s_count[1][tid] + s_count[2][tid];
    a.word[1][(int)blockIdx.x * kSearchTile + count] = key;
    if (i < a.n_q) a.slot[1][i] = count;
}

__global__ void __launch_bounds__(kSearchTile) sort_search_kernel(SortArgs a) {
    __shared__ __attribute__((aligned(16))) int s_key[kSearchGroup * kSearchTile];
    const int tiles = (a.n_q + kSearchTile - 1) / kSearchTile, t0 = (int)blockIdx.y * kSearchGroup, nt = min(kSearchGroup, tiles - t0);
    const int tid = threadIdx.x, own = blockIdx.x, i = own * kSearchTile + tid;
    for (int c = tid; c < nt * (kSearchTile / 4); c += kSearchTile)
        reinterpret_cast<int4*>(s_key)[c] = reinterpret_cast<const int4*>(a.word[1] + (size_t)t0 * kSearchTile)[c];
    const int key = i < a.n_q ? slot_word(a.tokens, a.q_idx, i, a.t_kv, a.vocab, a.vocab) : 0;
    int count = i < a.n_q && own >= t0 && own < t0 + nt ? a.slot[1][i] : 0;
    __syncthreads();
    // words below the slot's; of the tiles in front of its own, also the same word
    constexpr int kAtOnce = 4;
    for (int t = 0; t < nt; t += kAtOnce) {
        int at[kAtOnce], limit[kAtOnce];
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) {
            at[k] = 0;
            limit[k] = t + k < nt && t0 + t + k != own ? key + (t0 + t + k < own) : -1;         // -1: none
        }
#pragma unroll
        for (int step = kSearchTile / 2; step > 0; step /= 2)
#pragma unroll
            for (int k = 0; k < kAtOnce; ++k) at[k] += s_key[min(t + k, nt - 1) * kSearchTile + at[k] + step - 1] < limit[k] ? step : 0;
#pragma unroll
        for (int k = 0; k < kAtOnce; ++k) count += at[k] + (s_key[min(t + k, nt - 1) * kSearchTile + at[k]] < limit[k]);
    }
    if (i < a.n_q) a.hist[(size_t)blockIdx.y * a.n_q + i] = count;
}

// Slots to their places.
__global__ void __launch_bounds__(256) sort_place_kernel(SortArgs a) {
    const int i = (int)(blockIdx.x * 256 + threadIdx.x);
    if (i >= a.n_q) return;
    uint32_t at = 0;
#pragma unroll 8
    for (int y = 0; y < a.blocks; ++y) at += a.hist[(size_t)y * a.n_q + i];
    a.word[0][at] = slot_word(a.tokens, a.q_idx, i, a.t_kv, a.vocab, a.vocab);
    a.slot[0][at] = i;
}

__device__ __forceinline__ uint32_t load_lds(const uint32_t* p) { return *(const volatile uint32_t*)p; }
__device__ __forceinline__ void store_lds(uint32_t* p, uint32_t v) { *(volatile uint32_t*)p = v; }

// Ranks of this wavefront's keys among its own keys of the same digit, in order (round by round, lane by lane); count[digit][wave] ends up
// as the number of its keys of each digit.  count must be zero.  Keys of one digit find each other by comparing the digits' bits over the wavefront.
template <int R>
__device__ __forceinline__ void rank_digits(const uint32_t (&key)[R], uint32_t (&rank)[R], uint32_t* count, int shift, int bits, int wave, int lane) {
    const uint32_t mask = (1u << bits) - 1;
    const unsigned long long below = (1ull << lane) - 1;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t d = (key[r] >> shift) & mask;
        unsigned long long same = ~0ull;
        for (int b = 0; b < bits; ++b) {
            const bool one = (d >> b) & 1;
            const unsigned long long votes = __ballot(one);
            same &= one ? votes : ~votes;
        }
        uint32_t* at = count + d * kSortWaves + wave;
        const uint32_t before = load_lds(at);
        rank[r] = before + __popcll(same & below);
        __builtin_amdgcn_wave_barrier();
        if ((same & below) == 0) store_lds(at, before + __popcll(same));
        __builtin_amdgcn_wave_barrier();
    }
}

// Exclusive prefix sums of values held `per` to a thread (consecutive in LDS), in place; the workgroup has kSortThreads threads.
__device__ __forceinline__ void scan_lds(uint32_t* v, int n, uint32_t* wave_sums) {
    const int per = (n + kSortThreads - 1) / kSortThreads, t0 = threadIdx.x * per, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    uint32_t sum = 0;
    for (int i = t0; i < min(t0 + per, n); ++i) sum += v[i];
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_up(upto, o);
        if (lane >= o) upto += u;
    }
    if (lane == 63) wave_sums[wave] = upto;
    __syncthreads();
    uint32_t base = upto - sum;
    for (int w = 0; w < wave; ++w) base += wave_sums[w];
    for (int i = t0; i < min(t0 + per, n); ++i) {
        const uint32_t x = v[i];
        v[i] = base;
        base += x;
    }
    __syncthreads();
}

// Sort by digits, least significant first.  src: the list that the pass reads, -1 = the slots themselves.
__device__ __forceinline__ int sort_key(const SortArgs& a, int src, int i) {
    if (i >= a.n_q) return a.vocab;
    return src < 0 ? slot_word(a.tokens, a.q_idx, i, a.t_kv, a.vocab, a.vocab) : a.word[src][i];
}

__global__ void __launch_bounds__(kSortThreads) sort_hist_kernel(SortArgs a, int src, int shift) {
    __shared__ uint32_t s_bin[1 << kDigitBits];
    const int bins = 1 << a.bits;
    for (int i = threadIdx.x; i < bins; i += kSortThreads) s_bin[i] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kSortBlock / kSortThreads; ++r) {
        const int i = (int)blockIdx.x * kSortBlock + r * kSortThreads + (int)threadIdx.x;
        if (i < a.n_q) atomicAdd(&s_bin[(sort_key(a, src, i) >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += kSortThreads) a.hist[(size_t)i * a.blocks + blockIdx.x] = s_bin[i];
}

__global__ void __launch_bounds__(kSortThreads) sort_scan_kernel(SortArgs a) {
    __shared__ uint32_t s_v[8 * kSortThreads], s_sums[kSortWaves], s_total;
    const int n = a.blocks << a.bits;
    uint32_t base = 0;
    for (int n0 = 0; n0 < n; n0 += 8 * kSortThreads) {
        const int m = min(n - n0, 8 * kSortThreads);
        for (int i = threadIdx.x; i < m; i += kSortThreads) s_v[i] = a.hist[n0 + i];
        __syncthreads();
        const uint32_t last = threadIdx.x == 0 ? s_v[m - 1] : 0;
        scan_lds(s_v, m, s_sums);
        if (threadIdx.x == 0) s_total = s_v[m - 1] + last;
        for (int i = threadIdx.x; i < m; i += kSortThreads) a.hist[n0 + i] = base + s_v[i];
        __syncthreads();
        base += s_total;
    }
}

__global__ void __launch_bounds__(kSortThreads) sort_scatter_kernel(SortArgs a, int src, int dst, int shift) {
    constexpr int R = kSortBlock / kSortThreads;
    __shared__ uint32_t s_count[kSortWaves << kDigitBits];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, at0 = (int)blockIdx.x * kSortBlock + wave * (64 * R) + lane;
    const int bins = 1 << a.bits;
    for (int i = threadIdx.x; i < bins * kSortWaves; i += kSortThreads) s_count[i] = 0;
    uint32_t key[R], rank[R];
#pragma unroll
    for (int r = 0; r < R; ++r) key[r] = sort_key(a, src, at0 + r * 64);
    __syncthreads();
    rank_digits<R>(key, rank, s_count, shift, a.bits, wave, lane);
    __syncthreads();
    for (int d = threadIdx.x; d < bins; d += kSortThreads) {
        uint32_t base = a.hist[(size_t)d * a.blocks + blockIdx.x];
        for (int w = 0; w < kSortWaves; ++w) {
            const uint32_t n = s_count[d * kSortWaves + w];
            s_count[d * kSortWaves + w] = base;
            base += n;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = at0 + r * 64;
        if (i >= a.n_q) continue;       // slots past the end stand behind every other one of their digit
        const uint32_t to = s_count[((key[r] >> shift) & (bins - 1)) * kSortWaves + wave] + rank[r];
        a.word[dst][to] = (int)key[r];
        a.slot[dst][to] = src < 0 ? i : a.slot[src][i];
    }
}

// ------------------------------------------------------------------------------------------
// Sums over the sorted list.  It is cut into pieces of `piece` positions, and a wavefront takes one piece and 512 columns (16 bytes a
// lane): every wavefront has the same work however often a word occurs.  The sum of a word that lies within
// one piece is final; one that crosses pieces leaves a partial sum for each (first_part: the word that began in an earlier
// piece, last_part: the one that goes on in the next), which embed_join_kernel adds up in order.
// Bound by memory: every row of dx once, every row of dtable once (overwriting) or the present ones twice (adding).
constexpr int kSumUnroll = 8, kFillRows = 16;
constexpr int kFillMost = 1 << 20;              // workgroups that fill, at most

struct SumArgs {
    const int32_t *word, *slot;
    const uint4* dx;
    uint4* dtable;
    float4* part;            // [pieces][2][chunks][2]: partial sums, 8 floats a chunk of 16 bytes of bf16
    int n_q, vocab, chunks, strips, piece, pieces, add;
    int sum_blocks;          // workgroups that sum; the others fill absent rows with zeros
    float scale;
};

// first position of the sorted list that holds a word >= w
__device__ __forceinline__ int lower_bound(const int32_t* word, int n, int w) {
    int lo = 0, hi = n;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (word[mid] < w) lo = mid + 1; else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ void put_row(const SumArgs& a, int word, int c, const float (&s)[8]) {
    uint4* to = a.dtable + (size_t)word * a.chunks + c;
    float o[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) o[k] = a.scale * s[k];
    if (a.add) {
        const uint4 old = *to;
        const uint32_t p[4] = {old.x, old.y, old.z, old.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float u, v;
            unpack2(p[k], u, v);
            o[2 * k] += u;
            o[2 * k + 1] += v;
        }
    }
    *to = uint4{pack2(o[0], o[1]), pack2(o[2], o[3]), pack2(o[4], o[5]), pack2(o[6], o[7])};
}

__device__ __forceinline__ void put_part(const SumArgs& a, int piece, int last, int c, const float (&s)[8]) {
    float4* to = a.part + ((size_t)(2 * piece + last) * a.chunks + c) * 2;
    to[0] = float4{s[0], s[1], s[2], s[3]};
    to[1] = float4{s[4], s[5], s[6], s[7]};
}

__global__ void __launch_bounds__(256) embed_sum_kernel(SumArgs a) {
    const int wave = uniform((int)threadIdx.x >> 6), lane = threadIdx.x & 63, n = a.n_q;
    if ((int)blockIdx.x >= a.sum_blocks) {
        for (int row0 = (((int)blockIdx.x - a.sum_blocks) * 4 + wave) * kFillRows; row0 < a.vocab; row0 += kFillMost * 4 * kFillRows) {
            const int row = row0 + lane;
            bool absent = false;
            if (lane < kFillRows && row < a.vocab) {
                const int at = lower_bound(a.word, n, row);
                absent = at >= n || a.word[at] != row;
            }
            unsigned long long todo = __ballot(absent);
            while (todo) {
                const int r = __ffsll(todo) - 1;
                todo &= todo - 1;
                uint4* to = a.dtable + (size_t)(row0 + r) * a.chunks;
                for (int c = lane; c < a.chunks; c += 64) to[c] = uint4{0, 0, 0, 0};
            }
        }
        return;
    }
    const int task = (int)blockIdx.x * 4 + wave, piece = task / a.strips, c = (task - piece * a.strips) * 64 + lane;
    const int p0 = piece * a.piece;
    if (piece >= a.pieces) return;
    const bool on = c < a.chunks;
    const int at = min(p0 + lane, n - 1);
    const int my_word = a.word[at], my_slot = a.slot[at];
    const int count = __popcll(__ballot(lane < a.piece && p0 + lane < n && my_word < a.vocab));      // the slots without a word stand at the end
    if (count == 0) return;
    const int before = p0 > 0 ? a.word[p0 - 1] : -1, behind = p0 + count < n ? a.word[p0 + count] : -1;
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    bool began = before != __builtin_amdgcn_readlane(my_word, 0);       // the current word's first slot lies in this piece
    for (int i0 = 0; i0 < count; i0 += kSumUnroll) {
        uint4 v[kSumUnroll];
#pragma unroll
        for (int u = 0; u < kSumUnroll; ++u) {
            const int slot = __builtin_amdgcn_readlane(my_slot, min(i0 + u, count - 1));
            v[u] = on ? a.dx[(size_t)slot * a.chunks + c] : uint4{0, 0, 0, 0};
        }
#pragma unroll
        for (int u = 0; u < kSumUnroll; ++u) {
            const int i = i0 + u;
            if (i >= count) break;
            const uint32_t p[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float x, y;
                unpack2(p[k], x, y);
                s[2 * k] += x;
                s[2 * k + 1] += y;
            }
            const int word = __builtin_amdgcn_readlane(my_word, i);
            const int next = i + 1 < count ? __builtin_amdgcn_readlane(my_word, min(i + 1, 63)) : behind;
            if (word == next && i + 1 < count) continue;
            if (on) {
                if (!began) put_part(a, piece, 0, c, s);
                else if (word == next) put_part(a, piece, 1, c, s);
                else put_row(a, word, c, s);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) s[k] = 0;
            began = true;
        }
    }
}

// Sums that cross pieces: a workgroup per piece whose last word begins there and goes on, and 512 columns; each wavefront adds up a quarter of the
// word's partial sums.
__global__ void __launch_bounds__(256) embed_join_kernel(SumArgs a) {
    __shared__ float s_sum[3][8][64];
    const int wave = uniform((int)threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int piece = (int)blockIdx.x / a.strips, c = ((int)blockIdx.x - piece * a.strips) * 64 + lane;
    const int p0 = piece * a.piece, p1 = p0 + a.piece;
    if (p1 >= a.n_q) return;
    const int word = a.word[p1 - 1];
    if (word >= a.vocab || a.word[p1] != word || (p0 > 0 && a.word[p0 - 1] == word)) return;
    const int last = uniform((lower_bound(a.word, a.n_q, word + 1) - 1) / a.piece);     // piece that holds the word's last slot
    const int first = piece + 1 + (int)((long long)(last - piece) * wave / 4), end = piece + 1 + (int)((long long)(last - piece) * (wave + 1) / 4);
    const bool on = c < a.chunks;
    float s[8] = {0, 0, 0, 0, 0, 0, 0, 0};
    auto add = [&](const float4& u, const float4& v) __attribute__((always_inline)) {
        s[0] += u.x; s[1] += u.y; s[2] += u.z; s[3] += u.w;
        s[4] += v.x; s[5] += v.y; s[6] += v.z; s[7] += v.w;
    };
    auto part = [&](int p, int which) __attribute__((always_inline)) { return a.part + ((size_t)(2 * p + which) * a.chunks + (on ? c : 0)) * 2; };
    if (wave == 0) add(part(piece, 1)[0], part(piece, 1)[1]);
    for (int p = first; p < end; p += kSumUnroll) {
        float4 u[kSumUnroll], v[kSumUnroll];
#pragma unroll
        for (int k = 0; k < kSumUnroll; ++k) {
            const float4* from = part(min(p + k, end - 1), 0);
            u[k] = from[0];
            v[k] = from[1];
        }
#pragma unroll
        for (int k = 0; k < kSumUnroll; ++k)
            if (p + k < end) add(u[k], v[k]);
    }
    if (wave > 0) {
#pragma unroll
        for (int k = 0; k < 8; ++k) s_sum[wave - 1][k][lane] = s[k];
    }
    __syncthreads();
    if (wave > 0 || !on) return;
#pragma unroll
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int k = 0; k < 8; ++k) s[k] += s_sum[w][k][lane];
    put_row(a, word, c, s);
}

// Positions per piece: 64 (a wavefront's lanes hold the list), fewer where that leaves less than eight wavefronts to a compute unit.
static int sum_piece(const wlb_vocab_desc& d) {
    const long long strips = (d.hidden / 8 + 63) / 64;
    int piece = 64;
    while (piece > 8 && (d.n_q + piece - 1) / piece * strips < 8LL * compute_units()) piece /= 2;
    return piece;
}

struct EmbedLayout {
    size_t off_word[2], off_slot[2], off_hist, off_part, bytes;
    int passes, bits, blocks, piece, pieces;
    bool search;                     // sorted by search, `blocks` groups of tiles
};

static EmbedLayout embed_layout(const wlb_vocab_desc& d) {
    EmbedLayout L;
    int bits = 1;
    while (((unsigned)d.vocab >> bits) != 0) ++bits;             // keys 0 .. vocab
    L.passes = (bits + kDigitBits - 1) / kDigitBits;
    L.bits = (bits + L.passes - 1) / L.passes;
    L.search = d.n_q <= kSearchMost;
    const int per = L.search ? kSearchTile * kSearchGroup : kSortBlock;
    L.blocks = (d.n_q + per - 1) / per;
    L.piece = sum_piece(d);
    L.pieces = (d.n_q + L.piece - 1) / L.piece;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at += align_up(bytes, 256); return o; };
    for (int i = 0; i < 2; ++i) {
        const size_t list = sizeof(int32_t) * align_up(d.n_q, kSearchTile);
        L.off_word[i] = take(list);
        L.off_slot[i] = take(list);
    }
    L.off_hist = take(sizeof(uint32_t) * (L.search ? (size_t)L.blocks * d.n_q : (size_t)L.blocks << L.bits));
    L.off_part = take(sizeof(float) * 2 * (size_t)L.pieces * d.hidden);
    L.bytes = at;
    return L;
}

size_t embed_bwd_bytes(const wlb_vocab_desc& d) { return embed_layout(d).bytes; }

}  // namespace wlb

using namespace wlb;

extern "C" wlb_status wlb_embed_fwd(const wlb_vocab_desc* desc, const int32_t* tokens, const int32_t* q_idx, const void* table, void* x,
                                    void* stream) {
    if (wlb_status st = check_vocab(desc, "wlb_embed_fwd", 0)) return st;
    if (!tokens || !q_idx || !table || !x) return fail(WLB_ERR_INVALID_ARG, "wlb_embed_fwd: null pointer");
    if (misaligned(table, 16) || misaligned(x, 16) || misaligned(tokens, 4) || misaligned(q_idx, 4))
        return fail(WLB_ERR_INVALID_ARG, "wlb_embed_fwd: misaligned pointer");
    const int chunks = desc->hidden / 8;
    int lanes_log2 = 0;
    while ((1 << lanes_log2) < chunks && lanes_log2 < 8) ++lanes_log2;
    const int rows = (256 >> lanes_log2) * kLookupRows;
    const int most = (int)std::min((1LL << 23) * rows, (long long)desc->n_q);      // slots to a launch, which has fewer than 2^32 threads
    for (int first = 0; first < desc->n_q; first += most) {
        const int n = std::min(most, desc->n_q - first);
        embed_fwd_kernel<<<(n + rows - 1) / rows, 256, 0, (hipStream_t)stream>>>(tokens, q_idx + first, (const uint4*)table, (uint4*)x + (size_t)first * chunks, n,
                                                                                 desc->t_kv, desc->vocab, chunks, lanes_log2, desc->scale);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "lookup launch: %s", hipGetErrorString(e));
    return WLB_OK;
}

extern "C" wlb_status wlb_embed_bwd(const wlb_vocab_desc* desc, const int32_t* tokens, const int32_t* q_idx, const void* dx, void* dtable,
                                    void* workspace, size_t workspace_bytes, void* stream_) {
    if (wlb_status st = check_vocab(desc, "wlb_embed_bwd", WLB_VOCAB_ACCUMULATE)) return st;
    if (!tokens || !q_idx || !dx || !dtable || !workspace) return fail(WLB_ERR_INVALID_ARG, "wlb_embed_bwd: null pointer");
    if (misaligned(dx, 16) || misaligned(dtable, 16) || misaligned(tokens, 4) || misaligned(q_idx, 4) || misaligned(workspace, 256))
        return fail(WLB_ERR_INVALID_ARG, "wlb_embed_bwd: misaligned pointer");
    const wlb_vocab_desc& d = *desc;
    const EmbedLayout L = embed_layout(d);
    if (workspace_bytes < L.bytes) return fail(WLB_ERR_BUFFER_TOO_SMALL, "wlb_embed_bwd: workspace %zu < %zu bytes", workspace_bytes, L.bytes);
    hipStream_t stream = (hipStream_t)stream_;
    char* ws = (char*)workspace;
    SortArgs s;
    s.tokens = tokens; s.q_idx = q_idx;
    for (int i = 0; i < 2; ++i) {
        s.word[i] = (int32_t*)(ws + L.off_word[i]);
        s.slot[i] = (int32_t*)(ws + L.off_slot[i]);
    }
    s.hist = (uint32_t*)(ws + L.off_hist);
    s.n_q = d.n_q; s.t_kv = d.t_kv; s.vocab = d.vocab; s.passes = L.passes; s.bits = L.bits; s.blocks = L.blocks;
    if (d.n_q <= kDirectMost) {
        sort_direct_kernel<<<(d.n_q + kDirectSlots - 1) / kDirectSlots, kDirectMost, 0, stream>>>(s);
    } else if (L.search) {
        const int tiles = (d.n_q + kSearchTile - 1) / kSearchTile;
        sort_tile_kernel<<<tiles, 4 * kSearchTile, 0, stream>>>(s);
        sort_search_kernel<<<dim3(tiles, L.blocks), kSearchTile, 0, stream>>>(s);
        sort_place_kernel<<<(d.n_q + 255) / 256, 256, 0, stream>>>(s);
    } else {
        int src = -1;
        for (int pass = 0; pass < L.passes; ++pass) {
            const int dst = (L.passes - 1 - pass) & 1, shift = pass * L.bits;        // the last pass writes list 0
            sort_hist_kernel<<<L.blocks, kSortThreads, 0, stream>>>(s, src, shift);
            sort_scan_kernel<<<1, kSortThreads, 0, stream>>>(s);
            sort_scatter_kernel<<<L.blocks, kSortThreads, 0, stream>>>(s, src, dst, shift);
            src = dst;
        }
    }
    SumArgs a;
    a.word = s.word[0]; a.slot = s.slot[0]; a.n_q = d.n_q;
    a.dx = (const uint4*)dx; a.dtable = (uint4*)dtable; a.part = (float4*)(ws + L.off_part);
    a.vocab = d.vocab; a.chunks = d.hidden / 8; a.strips = (a.chunks + 63) / 64;
    a.piece = L.piece; a.pieces = L.pieces; a.add = d.flags & WLB_VOCAB_ACCUMULATE; a.scale = d.scale;
    a.sum_blocks = (int)(((long long)a.pieces * a.strips + 3) / 4);
    const int fill_blocks = a.add ? 0 : std::min((d.vocab + 4 * kFillRows - 1) / (4 * kFillRows), kFillMost);
    embed_sum_kernel<<<a.sum_blocks + fill_blocks, 256, 0, stream>>>(a);
    if (a.pieces > 1) embed_join_kernel<<<(unsigned)(a.pieces - 1) * a.strips, 256, 0, stream>>>(a);       // nothing goes on behind the last piece
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "lookup gradient launch: %s", hipGetErrorString(e));
    return WLB_OK;
}
