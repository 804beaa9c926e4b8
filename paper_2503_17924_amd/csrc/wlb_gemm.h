// Matrix products of the loss over the vocabulary: D[m][n] = sum_k P[m][k] * Q[n][k], bf16 operands, fp32 sums.
//
// Four wavefronts, each WM-th x WN-th part of a tile of TM x TN, in blocks of 16 x 16 x 32 (the power limit lets 16x16x32 MFMAs run at 1.73 - 1.80
// PFLOP/s on random operands and 32x32x16 ones at 1.64 - 1.68).  Operands move global -> LDS by buffer_load ... lds in
// steps of 64 along k, and LDS -> registers one 32-step ahead of the MFMAs.  An operand lies in memory either with k
// contiguous (rows of m or n: "K") or with m or n contiguous (rows of k: "M"); the second kind is read from LDS with transpose reads, so
// no operand is ever written transposed.  Wide tiles (256 x 256) take one workgroup to a compute unit and one wavefront to a SIMD: a wavefront's
// 128 x 128 part needs 16 KiB of LDS reads for 64 MFMAs, two thirds of what 8 wavefronts of 128 x 64 would read.  They are bound by the MFMA rate at
// the clock that the power limit leaves (16385 slots, 65536 words, hidden 4096: MFMAs busy 70 % of the cycles at 1.83 GHz; in the library's product 80 % at 1.66).  Narrow tiles (few slots) are bound by the table's bytes.
#pragma once
#include <type_traits>

#include "wlb_device.h"

namespace wlb {

constexpr int kStepK = 64;
constexpr int kTurn = 3;         // steps by which the starts of neighbouring tiles differ

// D[16x16] += A[16x32] * B[32x16], one wavefront.  Lane l supplies A[l%16][8*(l/16) .. +7] and B[8*(l/16) .. +7][l%16];
// accumulator register r of lane l is D[(l/16)*4 + r][l%16].
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }

// Place of 16-byte chunk cc of row r in an LDS tile of kind M: a transpose read takes 8 rows (r % 4, and 8 apart) x 2 chunks at a time, which
// this puts on 16 different chunks of 256 bytes.
__device__ __forceinline__ int swz_m(int r, int cc) { return cc ^ (((r & 3) << 2) | (((r >> 3) & 1) << 1)); }
constexpr int kOutOfRange = (int)0xfffffff0u;      // a lane offset at which every buffer load returns 0
constexpr uint32_t kMaxRecords = 0xffffffe0u;

template <int WM_, int WN_, int BM_, int BN_, bool MP_, bool MQ_>
struct GemmShape {
    static constexpr int WM = WM_, WN = WN_, BM = BM_, BN = BN_;         // wavefronts, and blocks of 16 of a wavefront
    static constexpr bool MP = MP_, MQ = MQ_;                            // operand kinds: m / n contiguous in memory
    static constexpr int TM = WM * BM * 16, TN = WN * BN * 16;
    static constexpr int P_BYTES = TM * kStepK * 2, Q_BYTES = TN * kStepK * 2, STAGE = P_BYTES + Q_BYTES;
    static constexpr bool RING = TM == 256 && TN == 256;
    // Three where both operands are of kind K: bound by the latency of the copies (33 slots, 32768 words, hidden 1024: D 13.5 us, with two 16.7; statistics of 128
    // slots, 50000 words, hidden 1536: 58 and 65).  dX waits for memory that dE has just written (45 slots, 65536 words, hidden 2048: 80 us, with two 77.5),
    // and dE keeps two workgroups to a compute unit (66 us, with three buffers and one 100).
    static constexpr int stages() { return !MP && !MQ && 3 * STAGE + 4 * OUT_WAVE <= 163840 ? 3 : 2; }
    // a wavefront's output on its way to memory: 32 rows of its bf16 values, or of 64 floats where sums are kept in parts
    static constexpr int OUT_WAVE = RING || (MP && !MQ) ? 8192 : BM * 1024;
    // five LDS slots of one operand's tile, one of them free for the output at an item's end; or STAGES buffers of both tiles, and the output
    static constexpr int STAGES = RING ? 2 : stages();
    static constexpr int LDS_BYTES = RING ? 5 * P_BYTES : STAGES * STAGE + 4 * OUT_WAVE;
    static constexpr int PER_CU = LDS_BYTES > 81920 || TN >= 128 && !MQ ? 1 : 2;        // workgroups to a compute unit
    static_assert(WM * WN == 4, "four wavefronts");
    static_assert(LDS_BYTES <= 163840, "LDS of a compute unit");
};

// A piece of work of a workgroup: a tile, and which part of k.
struct GemmItem {
    int tm, tn;
    int k0, depth;              // first k and how many (0: the product is 0)
    int part;                   // -1: the whole sum, else where its fp32 partial sum goes
};

// Distribution of the tiles of an ntm x ntn grid over the launch.  Whole tiles go round after round to the workgroups; those of a last round that would not
// fill the launch are divided along k, so that all workgroups share them, and leave partial sums that a second launch joins.  Workgroup b runs on
// XCD b % 8; each XCD takes a consecutive share of the tiles in bands of kBand tiles along n, so that the workgroups that run side by
// side on it share kBand operand tiles along n and a few along m in its L2.
constexpr int kBand = 8, kMaxParts = 128;
// In steps: an item's end (its sums go out while nothing else runs), and what a part costs the join, with its write and read of 256 KiB, in tenths.
constexpr int kEndSteps = 6, kJoinSteps = 4;
struct GemmGrid {
    int ntm, ntn, depth, workgroups, whole, left, parts;
    // part_steps: a divided tile's part has at least this many steps.  rounds: how many the parts may take; with one, tiles are divided wherever they can be,
    // with more where it pays: 160 tiles of 512 steps on 256 workgroups take 518 steps, in 3 parts each 2 * (171 + 6) and the join's 52.
    __device__ __forceinline__ GemmGrid(int ntm_, int ntn_, int depth_, int workgroups_, int part_steps, int rounds) : ntm(ntm_), ntn(ntn_), depth(depth_), workgroups(workgroups_) {
        const int tiles = ntm * ntn, steps = (depth + kStepK - 1) / kStepK, most = min(kMaxParts, steps / part_steps);
        left = uniform(tiles % workgroups);
        parts = 1;
        int least = rounds > 1 ? steps + kEndSteps : 1 << 30;
        for (int r = 1; left > 0 && r <= rounds; ++r) {
            const int p = min(uniform(r * workgroups / left), most);
            if (p < 2) continue;
            const int cost = r * (uniform(steps / p) + kEndSteps) + uniform(left * p / 10) + kJoinSteps;
            if (cost < least) { least = cost; parts = p; }
        }
        if (parts == 1) left = 0;
        whole = tiles - left;
    }
    __device__ __forceinline__ void place(int t, GemmItem& it) const {
        const int band = t / (kBand * ntm), high = min(kBand, ntn - band * kBand);
        t -= band * kBand * ntm;
        const int tm = t / high;
        it.tm = uniform(tm);            // divisions leave scalars in vector registers
        it.tn = uniform(band * kBand + (t - tm * high));
    }
    // item `round` of workgroup b; false: there is none
    __device__ __forceinline__ bool item(int b, int round, GemmItem& it) const {
        it.tm = it.tn = 0;
        const int x = b % kLists, i = b / kLists, side = workgroups / kLists;
        const int per = (whole + kLists - 1) / kLists, mine = round * side + i, t = x * per + mine;
        it.k0 = 0; it.depth = depth; it.part = -1;
        const int rounds = (per + side - 1) / side;
        if (round < rounds) {
            if (mine < per && t < whole) { place(t, it); return true; }
            if (round < rounds - 1 || left == 0) return false;
            round = rounds;                          // no whole tile in the last round
        }
        const int u = (round - rounds) * workgroups + x * side + i;
        if (u >= left * parts) return false;
        const int part = u / left, steps = (depth + kStepK - 1) / kStepK;
        place(whole + u - part * left, it);
        const int s0 = (int)((long long)steps * part / parts), s1 = (int)((long long)steps * (part + 1) / parts);
        it.k0 = uniform(s0 * kStepK);
        it.depth = uniform(min(depth, s1 * kStepK) - s0 * kStepK);
        it.part = uniform((u - part * left) * parts + part);
        return true;
    }
};

// An operand's part of a tile, as the caller gives it.
struct GemmOperand {
    const void* at;             // first element of the tile at the first k
    int valid;                  // rows or columns of the tile that exist
    const int32_t* list;        // kind K: numbers of the rows counted from `at`, or null
};

// Copies of one operand's tile.  T: its width (rows of kind K, columns of kind M).
template <int T, bool M>
struct TileCopy {
    static constexpr int N = T * kStepK * 2 / 1024 / 4;             // 1 KiB instructions per wavefront and step
    static constexpr int CH = M ? T / 8 : kStepK / 8;               // 16-byte chunks per LDS row
    static constexpr int RPI = 64 / CH;                         // LDS rows per instruction
    static_assert(N >= 1, "tile too narrow");
    int voff[N];
    BufRsrc rs;
    uint64_t base;
    uint32_t row_bytes;
    int wave, lane, left, turn;                                 // k that exist from this step's start on; where steps go on at k = 0, or 0

    __device__ __forceinline__ int row_of(int n) const { return (wave * N + n) * RPI + lane / CH; }
    __device__ __forceinline__ int chunk_of(int n) const { return M ? swz_m(row_of(n), lane % CH) : swz<8>(row_of(n), lane % CH); }
    // ld: elements between rows
    __device__ __forceinline__ void init(long long ld, int wave_, int lane_) {
        row_bytes = (uint32_t)(ld * 2);
        wave = wave_;
        lane = lane_;
    }
    __device__ __forceinline__ void tile(const GemmOperand& o) {
        base = (uint64_t)(uintptr_t)o.at;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int row = row_of(n), chunk = chunk_of(n);
            const bool on = (M ? chunk * 8 : row) < o.valid;
            uint32_t from = (uint32_t)row;
            if (!M && o.list) from = on ? (uint32_t)o.list[row] : 0u;
            voff[n] = on ? (int)(from * row_bytes + chunk * 16) : kOutOfRange;
        }
    }
    // the tile's first step, of `depth` along k, `start` steps from k = 0 (only where depth is whole steps); on = false: nothing is loaded
    __device__ __forceinline__ void first(int depth, bool on, int start = 0) {
        turn = start ? depth : 0;
        rs.r[0] = uniform((int)(uint32_t)base);
        rs.r[1] = uniform((int)(uint32_t)((base >> 32) & 0xffffu));
        rs.r[2] = on ? (int)kMaxRecords : 0;
        rs.r[3] = 0x00020000;
        left = depth;
        if (start) move(start * kStepK);
    }
    __device__ __forceinline__ void move(int k) {
        const uint64_t a = (((uint64_t)(uint32_t)rs.r[1] << 32) | (uint32_t)rs.r[0]) + (uint64_t)((long long)k * (M ? row_bytes : 2u));
        rs.r[0] = (int)(uint32_t)a;
        rs.r[1] = (int)(uint32_t)(a >> 32);
        left -= k;
    }
    __device__ __forceinline__ void next() { move(turn && left == kStepK ? kStepK - turn : kStepK); }
    // in the last step of a tile: lanes whose k does not exist load zeros from here on
    __device__ __forceinline__ void cut() {
        if (left >= kStepK) return;
#pragma unroll
        for (int n = 0; n < N; ++n)
            if ((M ? row_of(n) : chunk_of(n) * 8) >= left) voff[n] = kOutOfRange;
    }
    __device__ __forceinline__ void issue(int n, uint32_t lds_tile) const { dma_issue_1k(rs.r, lds_tile + (uint32_t)(wave * N + n) * 1024u, voff[n], 0u); }
};

// Operand fragments of a wavefront out of LDS: B blocks of 16 rows (columns).
template <int T, int B, bool M>
struct Fragments {
    static constexpr int READS = M ? 2 * B : B, KN = kStepK / 32;
    uint32_t at[M ? B : KN];        // K: by 32-step, the blocks 16 rows apart; M: by block, the 32-steps 32 rows apart

    __device__ __forceinline__ void init(uint32_t tile, int first, int lane) {
        if (M) {
#pragma unroll
            for (int i = 0; i < B; ++i) {
                const int row = 8 * (lane / 16) + (lane % 16) / 4, chunk = (first + i) * 2 + (lane % 4) / 2;
                at[i] = tile + row * (T * 2) + swz_m(row, chunk) * 16 + (lane % 2) * 8;
            }
        } else {
            const int row = first * 16 + lane % 16;
#pragma unroll
            for (int kk = 0; kk < KN; ++kk) at[kk] = tile + row * (kStepK * 2) + swz<8>(row, 4 * kk + lane / 16) * 16;
        }
    }
    __device__ __forceinline__ void move(int bytes) {
#pragma unroll
        for (int i = 0; i < (M ? B : KN); ++i) at[i] += bytes;
    }
    // read r of READS of 32-step kk into f
    __device__ __forceinline__ void read(int r, int kk, bf16x8 (&f)[B]) const {
        if (M) {
            const int i = r / 2, h = r % 2;
            const bf16x4 v = lds_read_tr4_at(at[i] + kk * 32 * T * 2 + h * 4 * T * 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[i][4 * h + e] = v[e];
        } else {
            f[r] = *reinterpret_cast<const WLB_LDS bf16x8*>((uintptr_t)(at[kk] + r * (16 * kStepK * 2)));
        }
    }
};

// Work is a GemmGrid with, for an item, operands p(item) and q(item) and leading dimensions ldp, ldq.  done(gemm, item, ahead, lds) takes the sums of an
// item; lds: OUT_WAVE bytes for each wavefront; ahead: what done.load(gemm, item) returned in front of the item's steps (loads that would hold up its end).
// It returns a number of vector memory operations that each wavefront has certainly issued: the next item's first step need not wait for those.
template <class S>
struct Gemm {
    f32x4 acc[S::BM][S::BN];    // register r of lane l: m = 16 i + (l/16)*4 + r, n = 16 j + l%16 of the wavefront's part
    int wave, lane, wm, wn;
    uint32_t lds;
    TileCopy<S::TM, S::MP> cp;
    TileCopy<S::TN, S::MQ> cq;
    Fragments<S::TM, S::BM, S::MP> fp;
    Fragments<S::TN, S::BN, S::MQ> fq;
    static constexpr int NP = decltype(cp)::N, NQ = decltype(cq)::N, RP = decltype(fp)::READS, RQ = decltype(fq)::READS;

    // An item has STAGES steps at least (later ones may be zeros), so that the steps that many ahead of its last ones are the next item's first.
    static __device__ __forceinline__ int steps_of(const GemmItem& it) { return max((it.depth + kStepK - 1) / kStepK, S::STAGES); }

    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < S::BM; ++i)
#pragma unroll
            for (int j = 0; j < S::BN; ++j)
#pragma unroll
                for (int r = 0; r < 4; ++r) acc[i][j][r] = 0.f;
    }

    template <class Work, class Done>
    __device__ __forceinline__ void run(char* smem, const Work& work, const Done& done) {
        wave = uniform((int)threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        wm = wave % S::WM;
        wn = wave / S::WM;
        lds = (uint32_t)(uintptr_t)smem;
        cp.init(work.ldp, wave, lane);
        cq.init(work.ldq, wave, lane);
        if constexpr (S::RING) ring(work, done);
        else pair(work, done);
    }

    // A narrow tile's first step.  Rows of a table lie 2^n bytes apart more often than not, and tiles that all began at k = 0 would read the same 128 bytes of
    // every row at a time, which few of the memory's channels hold (64K rows of 4096 bytes: a plain read in this order 4.1 TB/s, 5.5 with starts spread).
    __device__ __forceinline__ int start_of(const GemmItem& it) const {
        if constexpr (S::MP || S::MQ) return 0;
        if (it.depth % kStepK != 0 || it.depth < S::STAGES * kStepK) return 0;
        return uniform(kTurn * it.tm % (it.depth / kStepK));
    }

    // Narrow tiles in STAGES LDS buffers of both operands.  Here too copies go on from one item to the next while sums go to memory.
    template <class Work, class Done>
    __device__ __forceinline__ void pair(const Work& work, const Done& done) {
        constexpr int BM = S::BM, BN = S::BN, KN = kStepK / 32, ST = S::STAGES;
        GemmItem it, next = {};
        if (!work.item((int)blockIdx.x, 0, it)) return;
        cp.tile(work.p(it));
        cq.tile(work.q(it));
        fp.init(lds, wm * BM, lane);
        fq.init(lds + S::P_BYTES, wn * BN, lane);
#pragma unroll
        for (int s = 0; s < ST; ++s) {
            if (s) { cp.next(); cq.next(); }
            else { cp.first(it.depth, true, start_of(it)); cq.first(it.depth, true, start_of(it)); }
            cp.cut();
            cq.cut();
#pragma unroll
            for (int n = 0; n < NP; ++n) cp.issue(n, lds + s * S::STAGE);
#pragma unroll
            for (int n = 0; n < NQ; ++n) cq.issue(n, lds + s * S::STAGE + S::P_BYTES);
        }
        bf16x8 a[2][BM], b[2][BN];
        wait_vmem_le<(ST - 1) * (NP + NQ)>();
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RP; ++r) fp.read(r, 0, a[0]);
#pragma unroll
        for (int r = 0; r < RQ; ++r) fq.read(r, 0, b[0]);
        int buffer = 0;                         // of this step
        for (int round = 1;; ++round) {
            const int steps = steps_of(it);
            const bool more = work.item((int)blockIdx.x, round, next);
            GemmOperand next_p = {}, next_q = {};
            if (more) { next_p = work.p(next); next_q = work.q(next); }
            const auto ahead = done.load(*this, it);
            clear();
            for (int s = 0; s < steps; ++s) {
                const uint32_t stage = lds + buffer * S::STAGE;
#pragma unroll
                for (int kk = 0; kk < KN; ++kk) {
                    const int then = (kk + 1) % KN;
                    if (then == 0) {
                        // the step's last operands are in registers and the next step's tiles in LDS, for every wavefront
                        wait_lds();
                        wait_vmem_le<(ST - 2) * (NP + NQ)>();
                        __syncthreads();
                        if (s + ST == steps) {
                            if (more) { cp.tile(next_p); cq.tile(next_q); }
                            const int start = more ? start_of(next) : 0;
                            cp.first(next.depth, more, start);
                            cq.first(next.depth, more, start);
                        } else {
                            cp.next();
                            cq.next();
                        }
                        cp.cut();
                        cq.cut();
                        const int on = buffer < ST - 1 ? 1 : 1 - ST;
                        fp.move(on * S::STAGE);
                        fq.move(on * S::STAGE);
                        buffer += on;
                    }
#pragma unroll
                    for (int x = 0; x < BM * BN || x < RP + RQ || (then == 0 && x < NP + NQ); ++x) {
                        // reads of the operands of the next 32-step, copies of the step STAGES on, MFMAs of this one
                        if (x < RQ) fq.read(x, then, b[then & 1]);
                        else if (x < RP + RQ) fp.read(x - RQ, then, a[then & 1]);
                        if (then == 0) {
                            if (x < NP) cp.issue(x, stage);
                            else if (x < NP + NQ) cq.issue(x - NP, stage + S::P_BYTES);
                        }
                        if (x < BM * BN) {
                            const int i = x / BN, j = x % BN;
                            acc[i][j] = mfma16(a[kk & 1][i], b[kk & 1][j], acc[i][j]);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            }
            done(*this, it, ahead, lds + ST * S::STAGE);
            wait_lds();
            if (!more) break;
            it = next;
        }
        wait_vmem();
    }

    // Wide tiles.  The operands' tiles P0 Q0 P1 Q1 .. go to five LDS slots in turn, and on without a break from one item to the next:
    // while an item's sums go to memory, the first two steps of the next are in LDS or on their way, and the slot that is left holds the output.  Copies
    // take half of the time that the vector memory path has (64 KiB of 128 a step), so they are spread over the step: four wavefronts that
    // issued all of them in one quarter of it waited for each other (10 % more time).  Step s copies P of s + 2 beside its first
    // 32-step, into the slot that Q of s - 1 left, and behind the step's barrier Q of s + 2 into the slot of its own P. 
    template <class Work, class Done>
    __device__ __forceinline__ void ring(const Work& work, const Done& done) {
        constexpr int BM = S::BM, BN = S::BN, SLOT = S::P_BYTES;
        static_assert(NP == 8 && NQ == 8 && BM * BN == 64 && RP + RQ <= 32, "where in a step the copies stand");
        GemmItem it, next;
        if (!work.item((int)blockIdx.x, 0, it)) return;
        cp.tile(work.p(it));
        cq.tile(work.q(it));
        cp.first(it.depth, true);
        cq.first(it.depth, true);
        fp.init(lds, wm * BM, lane);
        fq.init(lds + SLOT, wn * BN, lane);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s) { cp.next(); cq.next(); }
            cp.cut();
            cq.cut();
#pragma unroll
            for (int n = 0; n < NP; ++n) cp.issue(n, lds + 2 * s * SLOT);
#pragma unroll
            for (int n = 0; n < NQ; ++n) cq.issue(n, lds + (2 * s + 1) * SLOT);
        }
        bf16x8 a[2][BM], b[2][BN];
        wait_vmem_le<NP + NQ>();
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RP; ++r) fp.read(r, 0, a[0]);
#pragma unroll
        for (int r = 0; r < RQ; ++r) fq.read(r, 0, b[0]);
        const f32x4 zeros = {0.f, 0.f, 0.f, 0.f};
        int p_slot = 0, q_slot = 1;             // of this step's tiles
        int stores = 0;
        for (int round = 1;; ++round) {
            const int steps = steps_of(it);
            const bool more = work.item((int)blockIdx.x, round, next);
            const auto ahead = done.load(*this, it);
            GemmOperand next_p = {}, next_q = {};
            if (more) { next_p = work.p(next); next_q = work.q(next); }
            auto step = [&](int s, auto fresh) __attribute__((always_inline)) {       // fresh: the sums start here, behind the last item's stores
                if (s + 2 == steps) {
                    if (more) cp.tile(next_p);
                    cp.first(next.depth, more);
                } else {
                    cp.next();
                }
                cp.cut();
                const uint32_t to_p = lds + (p_slot == 0 ? 4 : p_slot - 1) * SLOT, to_q = lds + p_slot * SLOT;
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    if (kk == 1) {
                        // the step's last operands are in registers and the next step's tiles in LDS, for every wavefront
                        wait_lds();
                        if (fresh && stores >= 32) wait_vmem_le<NP + 32>();
                        else wait_vmem_le<NP>();
                        __syncthreads();
                        if (s + 2 == steps) {
                            if (more) cq.tile(next_q);
                            cq.first(next.depth, more);
                        } else {
                            cq.next();
                        }
                        cq.cut();
                        const int p_move = p_slot < 3 ? 2 : -3, q_move = q_slot < 3 ? 2 : -3;
                        fp.move(p_move * SLOT);
                        fq.move(q_move * SLOT);
                        p_slot += p_move;
                        q_slot += q_move;
                    }
#pragma unroll
                    for (int x = 0; x < 64; ++x) {
                        // reads of the operands of the next 32-step, copies, MFMAs of this one
                        if (x % 2 == 0) {
                            if (x / 2 < RQ) fq.read(x / 2, kk ^ 1, b[kk ^ 1]);
                            else if (x / 2 < RP + RQ) fp.read(x / 2 - RQ, kk ^ 1, a[kk ^ 1]);
                        }
                        if (kk == 1 && x % 5 == 1 && x < 40) cq.issue(x / 5, to_q);
                        if (kk == 0 && x % 8 == 3) cp.issue(x / 8, to_p);
                        const int i = x / BN, j = x % BN;
                        acc[i][j] = mfma16(a[kk][i], b[kk][j], fresh && kk == 0 ? zeros : acc[i][j]);
                        if (x % 2 == 1) __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };
            step(0, std::true_type{});
            for (int s = 1; s < steps; ++s) step(s, std::false_type{});
            // the next P goes to the slot used here: each wavefront's copies to the 8 KiB that are its own
            sums_ready();
            stores = done(*this, it, ahead, lds + (p_slot == 0 ? 4 : p_slot - 1) * SLOT);
            wait_lds();
            if (!more) break;
            it = next;
        }
        wait_vmem();
    }

    // A sum.  Wide tiles' lie in accumulation registers, which vector instructions cannot read: moving them one by one, by hand, keeps the compiler from
    // copying them all.  It does not see when they were written: sums_ready() comes first.
    __device__ __forceinline__ float sum(int i, int j, int r) const {
        if constexpr (!S::RING) return acc[i][j][r];
        float v;
        asm("v_accvgpr_read_b32 %0, %1" : "=v"(v) : "a"(acc[i][j][r]));
        return v;
    }
    __device__ __forceinline__ void sums_ready() const {
        if constexpr (!S::RING) return;
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_nop 15\n\ts_nop 7" ::: "memory");       // an MFMA's result: 11 wait states, 19 for one of 16 passes
        __builtin_amdgcn_sched_barrier(0);
    }

    // Rows of output through LDS, so that memory sees whole 256-byte pieces: 32 rows n at a time (16 where there are no more), `Bytes` = 2 (bf16: all of the
    // wavefront's values of a row) or 4 (fp32: up to 64 of them).  value(i, j, r) gives the values; put(n, m, bits, j) takes 16 bytes: n, m counted in the tile, n
    // in one of the two blocks from j on.
    // mend(j, set): before a bf16 block j leaves, the lane may set(m, value) of its row n = lane % 16, m counted in the wavefront's part.
    struct NoMend { template <class Set> __device__ __forceinline__ void operator()(int, Set) const {} };
    template <int Bytes, class V, class Put, class Mend = NoMend>
    __device__ __forceinline__ void rows_out(uint32_t room, V value, Put put, Mend mend = Mend{}) {
        constexpr int MOST = 256 / (16 * Bytes), G = S::BM < MOST ? S::BM : MOST, H = S::BN < 2 ? S::BN : 2;    // blocks of 16 m, of 16 n at a time
        constexpr int ROWB = G * 16 * Bytes, CH = ROWB / 16, RPI = 64 / CH;                      // bytes, chunks of a row; rows per pass
        static_assert(S::BM % G == 0 && S::BN % H == 0 && ROWB <= 256 && 16 * H % RPI == 0, "whole passes");
        const uint32_t mine = room + wave * S::OUT_WAVE;
        int l = lane;
        asm volatile("" : "+v"(l));         // addresses are made here: made in front of all items, they take registers that the steps need
#pragma unroll
        for (int j0 = 0; j0 < S::BN; j0 += H)
#pragma unroll
            for (int i0 = 0; i0 < S::BM; i0 += G) {
#pragma unroll
                for (int j = 0; j < H; ++j)
#pragma unroll
                    for (int i = 0; i < G; ++i) {
                        const int row = j * 16 + l % 16, byte = (i * 16 + (l / 16) * 4) * Bytes;
                        const uint32_t to = mine + row * ROWB + (((byte / 16) ^ (row & (CH - 1))) * 16) + byte % 16;
                        const float v0 = value(i0 + i, j0 + j, 0), v1 = value(i0 + i, j0 + j, 1), v2 = value(i0 + i, j0 + j, 2), v3 = value(i0 + i, j0 + j, 3);
                        if (Bytes == 2) *reinterpret_cast<WLB_LDS bf16x4*>((uintptr_t)to) = pack4(v0, v1, v2, v3);
                        else *reinterpret_cast<WLB_LDS f32x4*>((uintptr_t)to) = f32x4{v0, v1, v2, v3};
                        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);      // few values out of the accumulators at a time
                    }
                if (Bytes == 2 && G == S::BM) {
#pragma unroll
                    for (int j = 0; j < H; ++j)
                        mend(j0 + j, [&](int m, float v) __attribute__((always_inline)) {
                            const int row = j * 16 + l % 16;
                            *reinterpret_cast<WLB_LDS __bf16*>((uintptr_t)(mine + row * ROWB + (((m * 2 / 16) ^ (row & (CH - 1))) * 16) + m * 2 % 16)) = (__bf16)v;
                        });
                }
                asm volatile("" ::: "memory");      // LDS takes a wavefront's accesses in their order
#pragma unroll
                for (int t = 0; t < 16 * H / RPI; ++t) {
                    const int n = t * RPI + l / CH, c = l % CH;
                    const i32x4 v = *reinterpret_cast<const WLB_LDS i32x4*>((uintptr_t)(mine + n * ROWB + ((c ^ (n & (CH - 1))) * 16)));
                    put(wn * (S::BN * 16) + j0 * 16 + n, wm * (S::BM * 16) + i0 * 16 + c * 16 / Bytes, v, j0);
                }
                asm volatile("" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
            }
    }

    // The partial sums of a divided tile: [TN][256] floats, of which `rows` are read (wide tiles write them all: comparisons in front of 64 stores made the
    // compiler keep registers in memory).
    __device__ __forceinline__ void part_out(uint32_t room, float* to, int rows) {
        static_assert(S::OUT_WAVE == 8192, "32 rows of 64 floats");
        rows_out<4>(room, [&](int i, int j, int r) __attribute__((always_inline)) { return sum(i, j, r); },
                    [&](int n, int m, const i32x4& v, int) __attribute__((always_inline)) { if (S::RING || n < rows) *reinterpret_cast<i32x4*>(to + n * S::TM + m) = v; });
    }
};

}  // namespace wlb
