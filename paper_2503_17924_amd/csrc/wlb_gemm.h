// Matrix product of a workgroup: D[m][n] = sum_k P[m][k] * Q[n][k], bf16 operands, fp32 sums, for the loss over the vocabulary.
//
// Four wavefronts, each WM-th x WN-th part of a tile of TM x TN.  Operands move global -> LDS by buffer_load ... lds in
// steps of 64 along k, double buffered, and LDS -> registers one 16-step ahead of the MFMAs.  An operand lies in memory either with k
// contiguous (rows of m or n: "K") or with m or n contiguous (rows of k: "M"); the second kind is read from LDS with transpose reads, so
// no operand is ever written transposed.  Wide tiles take one workgroup to a compute unit and one wavefront to a SIMD: a wavefront's
// 128 x 128 part needs 8 KiB of LDS reads for 16 MFMAs (8192 flops a byte), half of what 8 wavefronts of 128 x 64 would read.
#pragma once
#include "wlb_device.h"

namespace wlb {

constexpr int kStepK = 64;
constexpr int kOutOfRange = (int)0xfffffff0u;      // a lane offset at which every buffer load returns 0
constexpr uint32_t kMaxRecords = 0xffffffe0u;

template <int WM_, int WN_, int BM_, int BN_, bool MP_, bool MQ_>
struct GemmShape {
    static constexpr int WM = WM_, WN = WN_, BM = BM_, BN = BN_;         // wavefronts, and blocks of 32 of a wavefront
    static constexpr bool MP = MP_, MQ = MQ_;                            // operand kinds: m / n contiguous in memory
    static constexpr int TM = WM * BM * 32, TN = WN * BN * 32;
    static constexpr int P_BYTES = TM * kStepK * 2, Q_BYTES = TN * kStepK * 2, STAGE = P_BYTES + Q_BYTES;
    // Five LDS slots of one operand's tile, or two buffers of both tiles
    static constexpr bool RING = P_BYTES == 32768 && Q_BYTES == 32768;
    static constexpr int LDS_BYTES = RING ? 5 * P_BYTES : 2 * STAGE;
    static_assert(LDS_BYTES >= 4 * 8192, "8 KiB of each wavefront's output on its way to memory");
    static_assert(WM * WN == 4, "four wavefronts");
};

// Copies of one operand's tile.  T: its width (rows of kind K, columns of kind M).
template <int T, bool M>
struct TileCopy {
    static constexpr int N = T * kStepK * 2 / 1024 / 4;         // 1 KiB instructions per wavefront and step
    static constexpr int CH = M ? T / 8 : 8;                    // 16-byte chunks per LDS row
    static constexpr int RPI = 64 / CH;                         // LDS rows per instruction
    static_assert(N >= 1, "tile too narrow");
    int voff[N];
    BufRsrc rs;
    uint64_t base;
    uint32_t step_bytes;

    static __device__ __forceinline__ int row_of(int wave, int n, int lane) { return (wave * N + n) * RPI + lane / CH; }
    static __device__ __forceinline__ int chunk_of(int row, int lane) {
        return M ? (lane % CH) ^ ((row & 3) << 2) : swz<8>(row, lane % 8);
    }
    // base: the tile's first element at k = 0; ld: elements between rows; valid: rows (K) or columns (M, rounded up to 8 by what lies there) inside the operand;
    // list: the rows' numbers (K), rows counted from `base`, or null
    __device__ __forceinline__ void init(const void* at, long long ld, int valid, const int32_t* list, int wave, int lane) {
        base = (uint64_t)(uintptr_t)at;
        step_bytes = M ? (uint32_t)(kStepK * ld * 2) : kStepK * 2;
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int row = row_of(wave, n, lane), chunk = chunk_of(row, lane);
            if (M) {
                voff[n] = chunk * 8 < valid ? (int)((uint32_t)row * (uint32_t)(ld * 2) + chunk * 16) : kOutOfRange;
            } else {
                const uint32_t from = row < valid ? (list ? (uint32_t)list[row] : (uint32_t)row) : 0u;
                voff[n] = row < valid ? (int)(from * (uint32_t)(ld * 2) + chunk * 16) : kOutOfRange;
            }
        }
    }
    // lanes whose k lies at or beyond `left` (k counted from the step's start): zeros from here on
    __device__ __forceinline__ void cut(int left, int wave, int lane) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const int row = row_of(wave, n, lane), chunk = chunk_of(row, lane);
            if ((M ? row : chunk * 8) >= left) voff[n] = kOutOfRange;
        }
    }
    // the descriptor of step s; steps past the last one load nothing
    __device__ __forceinline__ void seek(int s, int steps) {
        const uint64_t a = base + (uint64_t)s * step_bytes;
        rs.r[0] = (int)(uint32_t)a;
        rs.r[1] = (int)(uint32_t)((a >> 32) & 0xffffu);
        rs.r[2] = s < steps ? (int)kMaxRecords : 0;
        rs.r[3] = 0x00020000;
    }
    __device__ __forceinline__ void issue(int n, uint32_t lds_tile, int wave) const {
        dma_issue_1k(rs.r, lds_tile + (uint32_t)(wave * N + n) * 1024u, voff[n], 0u);
    }
};

// Operand fragments of a wavefront out of LDS: B blocks of 32 rows (columns).
template <int T, int B, bool M>
struct Fragments {
    static constexpr int READS = M ? 2 * B : B;
    uint32_t at[M ? B : 4];         // K: by 16-step, the blocks 4096 bytes apart; M: by block, the 16-steps 16 rows apart

    __device__ __forceinline__ void init(uint32_t tile, int first, int lane) {
        if (M) {
#pragma unroll
            for (int i = 0; i < B; ++i) {
                const int row = 8 * (lane / 32) + (lane % 16) / 4, chunk = (first + i) * 4 + 2 * ((lane / 16) & 1) + (lane % 4) / 2;
                at[i] = tile + row * (T * 2) + (chunk ^ ((row & 3) << 2)) * 16 + (lane % 2) * 8;
            }
        } else {
            const int row = first * 32 + lane % 32;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) at[kk] = tile + row * 128 + swz<8>(row, 2 * kk + lane / 32) * 16;
        }
    }
    __device__ __forceinline__ void move(int bytes) {
#pragma unroll
        for (int i = 0; i < (M ? B : 4); ++i) at[i] += bytes;
    }
    // read r of READS of 16-step kk into f
    __device__ __forceinline__ void read(int r, int kk, bf16x8 (&f)[B]) const {
        if (M) {
            const int i = r / 2, h = r % 2;
            const bf16x4 v = lds_read_tr4_at(at[i] + kk * 16 * T * 2 + h * 4 * T * 2);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[i][4 * h + e] = v[e];
        } else {
            f[r] = *reinterpret_cast<const WLB_LDS bf16x8*>((uintptr_t)(at[kk] + r * 4096));
        }
    }
};

// An operand as the caller gives it (the tile's own part of it).
struct GemmOperand {
    const void* at;             // first element of the tile at the first k
    long long ld;               // elements between rows
    int valid;                  // rows or columns of the tile that exist
    const int32_t* list;        // kind K: numbers of the rows, or null
};

template <class S>
struct Gemm {
    f32x16 acc[S::BM][S::BN];   // register r of lane l: m = 32 i + (r/4)*8 + (l/32)*4 + r%4, n = 32 j + l%32 of the wavefront's part
    int wave, lane, wm, wn;
    uint32_t lds;

    __device__ __forceinline__ void start(char* smem) {
        wave = uniform((int)threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        wm = wave % S::WM;
        wn = wave / S::WM;
        lds = (uint32_t)(uintptr_t)smem;
    }

    // acc = the product over k of [0, depth).  Ends with every copy landed and LDS free for other use.
    __device__ __forceinline__ void run(const GemmOperand& p, const GemmOperand& q, int depth) {
        constexpr int BM = S::BM, BN = S::BN;
#pragma unroll
        for (int i = 0; i < BM; ++i)
#pragma unroll
            for (int j = 0; j < BN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        const int steps = (depth + kStepK - 1) / kStepK, tail = depth % kStepK;
        if (steps == 0) return;
        TileCopy<S::TM, S::MP> cp;
        TileCopy<S::TN, S::MQ> cq;
        cp.init(p.at, p.ld, p.valid, p.list, wave, lane);
        cq.init(q.at, q.ld, q.valid, q.list, wave, lane);
        constexpr int NP = decltype(cp)::N, NQ = decltype(cq)::N;
        Fragments<S::TM, BM, S::MP> fp;
        Fragments<S::TN, BN, S::MQ> fq;
        if constexpr (S::RING) {
            ring(cp, cq, fp, fq, steps, tail);
            return;
        }
        fp.init(lds, wm * BM, lane);
        fq.init(lds + S::P_BYTES, wn * BN, lane);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s == steps - 1 && tail) { cp.cut(tail, wave, lane); cq.cut(tail, wave, lane); }
            cp.seek(s, steps);
            cq.seek(s, steps);
#pragma unroll
            for (int n = 0; n < NP; ++n) cp.issue(n, lds + s * S::STAGE, wave);
#pragma unroll
            for (int n = 0; n < NQ; ++n) cq.issue(n, lds + s * S::STAGE + S::P_BYTES, wave);
        }
        bf16x8 a[2][BM], b[2][BN];
        wait_vmem_le<NP + NQ>();
        __syncthreads();
#pragma unroll
        for (int r = 0; r < decltype(fp)::READS; ++r) fp.read(r, 0, a[0]);
#pragma unroll
        for (int r = 0; r < decltype(fq)::READS; ++r) fq.read(r, 0, b[0]);
        for (int s = 0; s < steps; ++s) {
            const uint32_t stage = lds + (s & 1) * S::STAGE;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                constexpr int RP = decltype(fp)::READS, RQ = decltype(fq)::READS;
                if (kk == 3) {
                    // the step's last operands are in registers and the next step's tiles in LDS, for every wavefront
                    wait_lds();
                    wait_vmem();
                    __syncthreads();
                    if (s + 2 == steps - 1 && tail) { cp.cut(tail, wave, lane); cq.cut(tail, wave, lane); }
                    cp.seek(s + 2, steps);
                    cq.seek(s + 2, steps);
                    const int flip = (s & 1) ? -S::STAGE : S::STAGE;
                    fp.move(flip);
                    fq.move(flip);
                }
#pragma unroll
                for (int x = 0; x < BM * BN || x < RP + RQ || (kk == 3 && x < NP + NQ); ++x) {
                    // reads of the operands of the next 16-step, copies of the step after the next, MFMAs of this one
                    if (x < RQ) fq.read(x, (kk + 1) & 3, b[(kk + 1) & 1]);
                    else if (x < RP + RQ) fp.read(x - RQ, (kk + 1) & 3, a[(kk + 1) & 1]);
                    if (kk == 3) {
                        if (x < NP) cp.issue(x, stage, wave);
                        else if (x < NP + NQ) cq.issue(x - NP, stage + S::P_BYTES, wave);
                    }
                    if (x < BM * BN) {
                        const int i = x / BN, j = x % BN;
                        acc[i][j] = mfma32(a[kk & 1][i], b[kk & 1][j], acc[i][j]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        wait_lds();
        wait_vmem();
        __syncthreads();
    }

    // The steps of a wide tile.  The operands' tiles P0 Q0 P1 Q1 .. go to five LDS slots in turn.  Copies take half of the time that the
    // vector memory path has (64 KiB of 128 a step), so they are spread over the step: four wavefronts that
    // issued all of them in one quarter of it waited for each other (72 % of the time).  Step s copies P of s + 2 beside its first three
    // 16-steps, into the slot that Q of s - 1 left, and behind the step's barrier Q of s + 2 into the slot of its own P.
    template <class CP, class CQ, class FP, class FQ>
    __device__ __forceinline__ void ring(CP& cp, CQ& cq, FP& fp, FQ& fq, int steps, int tail) {
        constexpr int BM = S::BM, BN = S::BN, NP = CP::N, NQ = CQ::N, SLOT = S::P_BYTES, RP = FP::READS, RQ = FQ::READS;
        static_assert(NP == 8 && NQ == 8 && BM * BN == 16, "where in a step the copies stand");
        fp.init(lds, wm * BM, lane);
        fq.init(lds + SLOT, wn * BN, lane);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (s == steps - 1 && tail) { cp.cut(tail, wave, lane); cq.cut(tail, wave, lane); }
            cp.seek(s, steps);
            cq.seek(s, steps);
#pragma unroll
            for (int n = 0; n < NP; ++n) cp.issue(n, lds + 2 * s * SLOT, wave);
#pragma unroll
            for (int n = 0; n < NQ; ++n) cq.issue(n, lds + (2 * s + 1) * SLOT, wave);
        }
        bf16x8 a[2][BM], b[2][BN];
        wait_vmem_le<NP + NQ>();
        __syncthreads();
#pragma unroll
        for (int r = 0; r < RP; ++r) fp.read(r, 0, a[0]);
#pragma unroll
        for (int r = 0; r < RQ; ++r) fq.read(r, 0, b[0]);
        int p_slot = 0, q_slot = 1;             // of this step's tiles
        for (int s = 0; s < steps; ++s) {
            if (s + 2 == steps - 1 && tail) cp.cut(tail, wave, lane);
            cp.seek(s + 2, steps);
            const uint32_t to_p = lds + (p_slot == 0 ? 4 : p_slot - 1) * SLOT, to_q = lds + p_slot * SLOT;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk) {
                if (kk == 3) {
                    // the step's last operands are in registers and the next step's tiles in LDS, for every wavefront
                    wait_lds();
                    wait_vmem_le<NP>();
                    __syncthreads();
                    if (s + 2 == steps - 1 && tail) cq.cut(tail, wave, lane);
                    cq.seek(s + 2, steps);
                    const int p_move = p_slot < 3 ? 2 : -3, q_move = q_slot < 3 ? 2 : -3;
                    fp.move(p_move * SLOT);
                    fq.move(q_move * SLOT);
                    p_slot += p_move;
                    q_slot += q_move;
                }
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    // reads of the operands of the next 16-step, copies, MFMAs of this one
                    if (x < RQ) fq.read(x, (kk + 1) & 3, b[(kk + 1) & 1]);
                    else if (x < RP + RQ) fp.read(x - RQ, (kk + 1) & 3, a[(kk + 1) & 1]);
                    if (kk == 3 && x % 2 == 1) cq.issue(x / 2, to_q, wave);
                    if (kk < 3 && (kk * 16 + x) % 6 == 2) cp.issue((kk * 16 + x) / 6, to_p, wave);
                    const int i = x / BN, j = x % BN;
                    acc[i][j] = mfma32(a[kk & 1][i], b[kk & 1][j], acc[i][j]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
        }
        wait_lds();
        wait_vmem();
        __syncthreads();
    }

    // Rows of output through LDS, so that memory sees whole 256-byte pieces: the wavefront's columns n of block j, `Bytes` = 2 (bf16: all
    // of the wavefront's 32 BM values of a row, 4 blocks at most) or 4 (fp32: two blocks at a time).  value(i, j, r) gives the values; put(n, m, ptr) takes
    // 16 bytes: n, m counted in the tile.  The caller's LDS must be free; each wavefront uses a part of its own.
    template <int Bytes, class V, class Put>
    __device__ __forceinline__ void rows_out(V value, Put put) {
        constexpr int G = Bytes == 2 ? (S::BM < 4 ? S::BM : 4) : (S::BM < 2 ? S::BM : 2);        // blocks of 32 m at a time
        constexpr int ROWB = G * 32 * Bytes, CH = ROWB / 16, RPI = 64 / CH;                      // bytes, chunks of a row; rows per pass
        static_assert(S::BM % G == 0 && ROWB <= 256, "8 KiB of a wavefront");
        const uint32_t mine = lds + wave * 8192;
#pragma unroll
        for (int j = 0; j < S::BN; ++j)
#pragma unroll
            for (int i0 = 0; i0 < S::BM; i0 += G) {
                const int row = lane % 32;
#pragma unroll
                for (int i = 0; i < G; ++i)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const int m = i * 32 + (r / 4) * 8 + (lane / 32) * 4, byte = m * Bytes;
                        const uint32_t to = mine + row * ROWB + (((byte / 16) ^ (row & (CH - 1))) * 16) + byte % 16;
                        const float v0 = value(i0 + i, j, r), v1 = value(i0 + i, j, r + 1), v2 = value(i0 + i, j, r + 2), v3 = value(i0 + i, j, r + 3);
                        if (Bytes == 2) *reinterpret_cast<WLB_LDS bf16x4*>((uintptr_t)to) = pack4(v0, v1, v2, v3);
                        else *reinterpret_cast<WLB_LDS f32x4*>((uintptr_t)to) = f32x4{v0, v1, v2, v3};
                    }
                wait_lds();
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int t = 0; t < 32 / RPI; ++t) {
                    const int n = t * RPI + lane / CH, c = lane % CH;
                    const i32x4 v = *reinterpret_cast<const WLB_LDS i32x4*>((uintptr_t)(mine + n * ROWB + ((c ^ (n & (CH - 1))) * 16)));
                    put(wn * (S::BN * 32) + j * 32 + n, wm * (S::BM * 32) + i0 * 32 + c * 16 / Bytes, v);
                }
                wait_lds();
                __builtin_amdgcn_wave_barrier();
            }
    }
};

}  // namespace wlb
