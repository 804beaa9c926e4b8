// Rotary positions of a rank's slots (wlb_rope_fwd / wlb_rope_bwd): rows of the query, key and value product divided into q, k and v, q and k turned
// by the place of their tokens in their documents, and the gradient of that.
//
// A pair (a, b) of a head becomes m (a cos t - b sin t, b cos t + a sin t), t = position * freq; the gradient turns back, by -t.  Bound by the bytes: every value is read and
// written once.  All heads of a row share its angles, so a workgroup finds the positions of its rows, forms their cosines and sines once, in LDS, and turns 16 values
// of a head to a thread.  The angle is formed in 64 bits, since at position 10^6 a float's step is 0.06, and its whole turns are taken out there.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "wlb_device.h"
#include "wlb_vocab.h"

namespace wlb {

struct RopeArgs {
    const __bf16* src[3];            // forward: the row's query, key and value heads; backward: dq, dk, dv
    __bf16* dst[3];
    long long src_row[3], dst_row[3];            // elements between rows
    const int32_t *q_idx, *cu;
    const double* freq;
    int n_q, t_kv, n_docs, hq, hkv, head_dim, rot;
    int turn_units, units;           // of a head that is turned; of a row
    float magnitude;
};

// A row's position, -1 for padding.  One wavefront: 64 offsets are looked at in a step.
__device__ __forceinline__ int row_position(const RopeArgs& a, int row) {
    const int g = a.q_idx[row];
    if ((unsigned)g >= (unsigned)a.t_kv) return -1;
    if (!a.cu) return g;
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = a.n_docs + 1;               // the first offset above g, the end of g's document, is in [lo, hi]
    while (lo < hi) {
        const int step = (hi - lo + 63) / 64, last = lo + lane * step + step - 1;
        const bool below = lo + lane * step < hi && a.cu[min(last, hi - 1)] <= g;
        const int c = __popcll(__ballot(below));     // pieces that lie below as a whole: offsets ascend
        const int from = min(lo + c * step, hi);
        hi = max(from, min(from + step - 1, hi));
        lo = from;
    }
    lo = uniform(lo);
    return lo == 0 || lo > a.n_docs ? -1 : g - a.cu[lo - 1];
}

// Values of a thread: pair i is (a[i], b[i]).
struct Pairs { float a[8], b[8]; };

// 16 values as two pieces of 8.
struct Raw { uint4 a, b; };

__device__ __forceinline__ float bf16_bits(uint32_t bits16) { return __builtin_bit_cast(float, bits16 << 16); }
__device__ __forceinline__ void floats(const uint4& v, float (&f)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { f[2 * i] = bf16_bits(w[i] & 0xffffu); f[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u); }
}
__device__ __forceinline__ uint4 bits(const float (&f)[8]) {
    const bf16x8 v = pack8(f[0], f[1], f[2], f[3], f[4], f[5], f[6], f[7]);
    return __builtin_bit_cast(uint4, v);
}

// Where the 16 values of a unit lie, and what is done with them.  A head that is turned has rot / 16 units of 8 pairs (rounded up), the rest of it and the value heads
// units of 16 values in turn.
struct Unit {
    int part, head, pair;            // 0 q, 1 k, 2 v; pair: the first, or -1: copied
    int at_a, at_b, n;               // first values of the two pieces in the head; how many of each (8 but at an odd end)
};
template <bool Half>
__device__ __forceinline__ Unit unit_of(const RopeArgs& a, int u) {
    Unit t;
    const int turned = (a.hq + a.hkv) * a.turn_units;
    if (u < turned) {
        const int h = u / a.turn_units, c = u - h * a.turn_units, pair_units = (a.rot + 15) / 16;
        t.part = h >= a.hq;
        t.head = h - (t.part ? a.hq : 0);
        if (c < pair_units) {
            t.pair = c * 8;
            t.at_a = Half ? c * 8 : c * 16;
            t.at_b = Half ? a.rot / 2 + c * 8 : c * 16 + 8;
            t.n = min(8, a.rot / 2 - c * 8);
            return t;
        }
        t.pair = -1;
        t.at_a = a.rot + (c - pair_units) * 16;
    } else {
        const int per = a.head_dim / 16, h = (u - turned) / per;
        t.part = 2;
        t.head = h;
        t.pair = -1;
        t.at_a = (u - turned - h * per) * 16;
    }
    t.at_b = t.at_a + 8;
    t.n = 8;
    return t;
}

// Whole: every piece is 8 values at a multiple of 8.  Otherwise (rotary_dim no multiple of 16) values are moved one by one, those that are not turned too: 16408 slots, 32 query
// and 8 key heads of 128, 128 of them turned 82 us, 30 500, 50 470, 98 500 (interleaved 85, 490, 460, 515).
template <bool Half, bool Whole, bool Back, int Rows>
__global__ void __launch_bounds__(256) rope_kernel(RopeArgs a) {
    extern __shared__ float2 s_turn[];                 // [Rows][rot / 2]
    __shared__ int s_pos[Rows];
    const int pairs = a.rot / 2, wave = uniform((int)threadIdx.x >> 6);
    for (int row0 = (int)blockIdx.x * Rows; row0 < a.n_q; row0 += (int)gridDim.x * Rows) {
        __syncthreads();
        for (int r = wave; r < Rows; r += 4) {
            const int p = row0 + r < a.n_q ? row_position(a, row0 + r) : -1;
            if ((threadIdx.x & 63) == 0) s_pos[r] = p;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < Rows * pairs; i += 256) {
            const int r = i / pairs, j = i - r * pairs;
            // turns, and what is left of them
            const double t = (double)s_pos[r] * a.freq[j] * 0.15915494309189533577;
            float s, c;
            sincospif(2.f * (float)(t - rint(t)), &s, &c);
            s_turn[i] = float2{a.magnitude * c, a.magnitude * (Back ? -s : s)};
        }
        __syncthreads();
        for (int i = threadIdx.x; i < Rows * a.units; i += 256) {
            const int r = i / a.units, row = row0 + r;
            if (row >= a.n_q) break;
            const Unit t = unit_of<Half>(a, i - r * a.units);
            const long long head = (long long)t.head * a.head_dim;
            const __bf16* from = a.src[t.part] + (long long)row * a.src_row[t.part] + head;
            __bf16* to = a.dst[t.part] + (long long)row * a.dst_row[t.part] + head;
            const bool real = s_pos[r] >= 0;
            const float2* turn = s_turn + r * pairs + t.pair;
            if constexpr (Whole) {
                Raw v = {uint4{0, 0, 0, 0}, uint4{0, 0, 0, 0}};
                if (real) {
                    v.a = *reinterpret_cast<const uint4*>(from + t.at_a);
                    v.b = *reinterpret_cast<const uint4*>(from + t.at_b);
                    if (t.pair >= 0) {
                        float x[8], y[8];
                        floats(v.a, x);
                        floats(v.b, y);
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            // half: pair k is (x[k], y[k]); interleaved: the neighbours of x, then those of y
                            float &p = Half ? x[k] : k < 4 ? x[2 * k] : y[2 * k - 8], &q = Half ? y[k] : k < 4 ? x[2 * k + 1] : y[2 * k - 7];
                            const float2 cs = turn[k];
                            const float e = p * cs.x - q * cs.y, f = q * cs.x + p * cs.y;
                            p = e;
                            q = f;
                        }
                        v.a = bits(x);
                        v.b = bits(y);
                    }
                }
                *reinterpret_cast<uint4*>(to + t.at_a) = v.a;
                *reinterpret_cast<uint4*>(to + t.at_b) = v.b;
            } else if (t.pair >= 0) {
                for (int k = 0; k < t.n; ++k) {
                    const int ia = Half ? t.at_a + k : t.at_a + 2 * k, ib = Half ? t.at_b + k : ia + 1;
                    const float p = real ? (float)from[ia] : 0.f, q = real ? (float)from[ib] : 0.f;
                    const float2 cs = turn[k];
                    to[ia] = (__bf16)(real ? p * cs.x - q * cs.y : 0.f);
                    to[ib] = (__bf16)(real ? q * cs.x + p * cs.y : 0.f);
                }
            } else {
                const int n = min(16, a.head_dim - t.at_a);
                for (int k = 0; k < n; ++k) to[t.at_a + k] = real ? from[t.at_a + k] : (__bf16)0.f;
            }
        }
    }
}

constexpr int kRopeGrid = 1 << 20;         // workgroups at most
constexpr int kRopeRows = 4;

template <bool Half, bool Whole, bool Back>
static void launch_rope(const RopeArgs& a, hipStream_t stream) {
    const bool many = a.n_q >= 8 * compute_units();
    const int rows = many ? kRopeRows : 1;
    const size_t lds = sizeof(float2) * (size_t)rows * (a.rot / 2);
    const int grid = std::min((a.n_q + rows - 1) / rows, kRopeGrid);
    if (many) rope_kernel<Half, Whole, Back, kRopeRows><<<grid, 256, lds, stream>>>(a);
    else rope_kernel<Half, Whole, Back, 1><<<grid, 256, lds, stream>>>(a);
}

static wlb_status check_rope(const wlb_rope_desc* d, const char* call, const int32_t* q_idx, const int32_t* cu, const double* freq) {
    if (!d) return fail(WLB_ERR_INVALID_ARG, "%s: null desc", call);
    if (d->n_q < 1 || d->t_kv < 1 || d->n_docs < 0 || d->hq < 1 || d->hkv < 0 || d->head_dim < 1)
        return fail(WLB_ERR_INVALID_ARG, "%s: n_q=%d t_kv=%d n_docs=%d hq=%d hkv=%d head_dim=%d", call, d->n_q, d->t_kv, d->n_docs, d->hq, d->hkv, d->head_dim);
    if (d->layout != WLB_ROPE_HALF && d->layout != WLB_ROPE_INTERLEAVED) return fail(WLB_ERR_INVALID_ARG, "%s: layout %d", call, d->layout);
    if (d->rotary_dim < 2 || d->rotary_dim % 2 != 0 || d->rotary_dim > d->head_dim)
        return fail(WLB_ERR_INVALID_ARG, "%s: rotary_dim=%d (even, 2 .. head_dim=%d)", call, d->rotary_dim, d->head_dim);
    if (!(d->magnitude > 0.0f) || !std::isfinite(d->magnitude)) return fail(WLB_ERR_INVALID_ARG, "%s: magnitude must be finite and > 0", call);
    if (d->n_q > (1 << 30) || d->n_docs > (1 << 30) || d->hq > 1024 || d->hkv > 1024)
        return fail(WLB_ERR_UNSUPPORTED, "%s: n_q=%d n_docs=%d hq=%d hkv=%d", call, d->n_q, d->n_docs, d->hq, d->hkv);
    if (d->head_dim % 16 != 0 || d->head_dim > 512) return fail(WLB_ERR_UNSUPPORTED, "%s: head_dim=%d (a multiple of 16 up to 512)", call, d->head_dim);
    if (d->row_stride < (int64_t)(d->hq + 2 * d->hkv) * d->head_dim || d->row_stride % 8 != 0 || d->row_stride >= (1ll << 31))
        return fail(WLB_ERR_INVALID_ARG, "%s: row_stride=%lld for rows of %d values (a multiple of 8)", call, (long long)d->row_stride, (d->hq + 2 * d->hkv) * d->head_dim);
    if (!q_idx || !freq || (d->n_docs > 0) != (cu != nullptr)) return fail(WLB_ERR_INVALID_ARG, "%s: null pointer (cu_seqlens_k goes with n_docs=%d)", call, d->n_docs);
    if (misaligned(q_idx, 4) || misaligned(cu, 4) || misaligned(freq, 8)) return fail(WLB_ERR_INVALID_ARG, "%s: misaligned pointer", call);
    return WLB_OK;
}

// row: the fused row; heads: q, k, v
static wlb_status rope(const wlb_rope_desc* desc, const char* call, const void* row, const void* const (&heads)[3], const int32_t* q_idx, const int32_t* cu, const double* freq,
                       bool back, hipStream_t stream) {
    if (wlb_status st = check_rope(desc, call, q_idx, cu, freq)) return st;
    const wlb_rope_desc& d = *desc;
    if (!row || !heads[0] || (d.hkv > 0) != (heads[1] != nullptr) || (d.hkv > 0) != (heads[2] != nullptr))
        return fail(WLB_ERR_INVALID_ARG, "%s: null pointer (keys and values go with hkv=%d)", call, d.hkv);
    if (misaligned(row, 16) || misaligned(heads[0], 16) || misaligned(heads[1], 16) || misaligned(heads[2], 16))
        return fail(WLB_ERR_INVALID_ARG, "%s: misaligned pointer", call);
    if (row == heads[0] && (d.hkv > 0 || d.row_stride != (int64_t)d.hq * d.head_dim))
        return fail(WLB_ERR_INVALID_ARG, "%s: in place only where rows hold the query heads alone", call);
    RopeArgs a = {};
    const int first[3] = {0, d.hq, d.hq + d.hkv}, count[3] = {d.hq, d.hkv, d.hkv};
    for (int i = 0; i < 3; ++i) {
        __bf16* in_row = (__bf16*)row + (size_t)first[i] * d.head_dim;
        a.src[i] = back ? (const __bf16*)heads[i] : in_row;
        a.dst[i] = back ? in_row : (__bf16*)heads[i];
        a.src_row[i] = back ? (long long)count[i] * d.head_dim : d.row_stride;
        a.dst_row[i] = back ? d.row_stride : (long long)count[i] * d.head_dim;
    }
    a.q_idx = q_idx; a.cu = cu; a.freq = freq;
    a.n_q = d.n_q; a.t_kv = d.t_kv; a.n_docs = d.n_docs; a.hq = d.hq; a.hkv = d.hkv; a.head_dim = d.head_dim; a.rot = d.rotary_dim; a.magnitude = d.magnitude;
    a.turn_units = (d.rotary_dim + 15) / 16 + (d.head_dim - d.rotary_dim + 15) / 16;
    a.units = (d.hq + d.hkv) * a.turn_units + d.hkv * (d.head_dim / 16);
    const bool half = d.layout == WLB_ROPE_HALF, whole = d.rotary_dim % 16 == 0;
    if (half) whole ? back ? launch_rope<true, true, true>(a, stream) : launch_rope<true, true, false>(a, stream)
                    : back ? launch_rope<true, false, true>(a, stream) : launch_rope<true, false, false>(a, stream);
    else whole ? back ? launch_rope<false, true, true>(a, stream) : launch_rope<false, true, false>(a, stream)
               : back ? launch_rope<false, false, true>(a, stream) : launch_rope<false, false, false>(a, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return fail(WLB_ERR_HIP, "rotary launch: %s", hipGetErrorString(e));
    return WLB_OK;
}

}  // namespace wlb

using namespace wlb;

extern "C" wlb_status wlb_rope_fwd(const wlb_rope_desc* desc, const void* qkv, const int32_t* q_idx, const int32_t* cu_seqlens_k, const double* freq, void* q, void* k,
                                   void* v, void* stream) {
    const void* const heads[3] = {q, k, v};
    return rope(desc, "wlb_rope_fwd", qkv, heads, q_idx, cu_seqlens_k, freq, false, (hipStream_t)stream);
}

extern "C" wlb_status wlb_rope_bwd(const wlb_rope_desc* desc, const void* dq, const void* dk, const void* dv, const int32_t* q_idx, const int32_t* cu_seqlens_k,
                                   const double* freq, void* dqkv, void* stream) {
    const void* const heads[3] = {dq, dk, dv};
    return rope(desc, "wlb_rope_bwd", dqkv, heads, q_idx, cu_seqlens_k, freq, true, (hipStream_t)stream);
}
