// Rotary embedding of packed q and k rows by one to four position axes (Sec. 3.2: the target LLM is unchanged; Qwen2.5-VL rotates
// the tokens of an image or a video by time, height and width), alone or on the way of a prompt's rows into the cache.
//
//   x'[j] = x[j] cos a - x[j + D/2] sin a,   x'[j + D/2] = x[j + D/2] cos a + x[j] sin a,   a = positions[axis(j)][t] * theta^(-2j/D)
//
// What bounds it: HBM, every row read once and written once; few rows: the chain launch -> positions -> rotation -> store.  So a warp
// forms the D/2 angles of its token once, with its first rows on their way, and turns all the rows it has of the token by them.  An
// angle is taken as a number of turns, position times frequency / 2 pi in fp64, whose whole part goes before the rest (half a turn at
// most) is rounded to fp32: 2^-26 of a turn, the fp64 part less than that up to positions of 2^22; then sine and cosine in fp32, and the
// products in fp32 with one rounding to bf16.  (Sines in fp64 cost two FP64 warps 400 cycles a token, as much as HBM needs for the 20
// rows of a 16/2-head model's token.)
// Measured, us of a call among others with changing inputs (floor at 6516 GB/s): 32768 tokens of 16/2 heads rotated 48.7 (46.4), 16000
// tokens of 40/40 heads appended 160 (151), 3344 of 28/4 rotated 11.1 (8.4) and appended 14.5 (9.5), 8 tokens rotated 2.9, 32 appended 3.5.
// Head size 64, back to back: 32768 tokens of 16/2 heads rotated 28.7 (23.2), 16000 of 40/40 appended 82 (75).
#include <cuda_bf16.h>
#include <algorithm>

#include "launch.cuh"
#include "rows.cuh"
#include "vispec_internal.h"

namespace vispec {

namespace {

constexpr int kRowWarps = 4, kWarpsPerSm = 16;     // of a block; of an SM, up to which a token is shared out

// The position axis of frequency j: sections' blocks, or dealt in turn (an axis that has its share leaves its turns to axis 0).
__device__ __forceinline__ int axis_of(int j, const RowsArgs& a) {
    if (a.interleaved) {
        const int x = j % a.n_axes;
        return j < a.n_axes * a.sections[x] ? x : 0;
    }
    int x = 0, end = a.sections[0];
    while (x + 1 < a.n_axes && j >= end) end += a.sections[++x];
    return x;
}

// cs[t]: (cos, sin) of two frequencies
__device__ __forceinline__ void rotate8(uint4& lo, uint4& hi, const float4* cs) {
    __nv_bfloat162* x = reinterpret_cast<__nv_bfloat162*>(&lo);
    __nv_bfloat162* y = reinterpret_cast<__nv_bfloat162*>(&hi);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const float4 c = cs[t];
        const float2 u = __bfloat1622float2(x[t]), w = __bfloat1622float2(y[t]);
        x[t] = __floats2bfloat162_rn(u.x * c.x - w.x * c.y, u.y * c.z - w.y * c.w);
        y[t] = __floats2bfloat162_rn(w.x * c.x + u.x * c.y, w.y * c.z + u.y * c.w);
    }
}

// Rows of a token: Hq of q (if any), Hkv of k (if any), Hkv of v (APPEND).  A warp has one token and one of `chunks` shares of its
// rows; D/16 lanes share a row, each with 8 elements of the lower half and the 8 they pair with.  A lane keeps its elements and goes
// through the rows, so that it reads its cosines and sines once, and nothing waits for another warp.  (32768 tokens of 16/2 heads: 73 us
// with a block's threads dealt over (token, row) items, whose divisions and conflicting reads of the sines took the L1 to 75 %;
// 54.5 with half a block to a token.)
template <int D, bool APPEND>
__global__ void __launch_bounds__(32 * kRowWarps, 8)
prompt_rows_kernel(const RowsArgs a, const RowMap map, const int chunks) {
    constexpr int TPR = D / 16, RP = 32 / TPR, U = 2, AP = D / 64;      // lanes to a row, rows at a time, times, angles of a lane
    __shared__ __align__(16) float4 cs[kRowWarps][D / 4];               // [frequency pair of the lane's four][lane of the row]
    extern __shared__ int cu[];                                          // APPEND: B + 1 ends of the sequences, their B lengths
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, rl = lane / TPR, c = lane % TPR;
    double freq[AP];
    int axis[AP];
#pragma unroll
    for (int x = 0; x < AP; ++x) {
        const int j = lane + 32 * x;
        freq[x] = exp2(-2.0 * (double)j / (double)D * a.log2_theta) * 0.15915494309189533577;          // turns per position
        axis[x] = a.n_axes ? axis_of(j, a) : 0;
    }
    pdl_wait();
    if constexpr (!APPEND) pdl_launch_dependents();    // (an append writes committed slots: what follows starts when it has ended)
    if constexpr (APPEND) {
        int* const len = cu + a.B + 1;
        for (int i = tid; i <= a.B; i += 32 * kRowWarps) {
            cu[i] = a.cu_len[i];
            if (i < a.B) len[i] = a.kv_len[i];
        }
        __syncthreads();
        bool sound = true;
        for (int i = tid; i < a.B; i += 32 * kRowWarps) sound &= cu[i] <= cu[i + 1];
        sound &= cu[0] >= 0 && cu[a.B] <= a.T;
        sound = __syncthreads_and(sound);
        if (!sound) {
            if (blockIdx.x == 0 && tid == 0) record_status(a.status, VISPEC_E_RANGE);
            return;
        }
        if (blockIdx.x == 0)
            for (int b = tid; b < a.B; b += 32 * kRowWarps) {
                const int S = len[b], n = cu[b + 1] - cu[b];
                if (S < 0 || S > a.S_max - n) record_status(a.status, VISPEC_E_RANGE);
                else if (a.kv_len_out) a.kv_len_out[b] = S + n;
            }
    }
    const int nq = a.q ? a.Hq : 0, nk = a.k ? a.Hkv : 0, rows = nq + nk + (APPEND ? a.Hkv : 0), share = (rows + chunks - 1) / chunks;
    const long long item = (long long)blockIdx.x * kRowWarps + warp, t = item / chunks;
    if (t >= a.T) return;
    const int r0 = (int)(item - t * chunks) * share, r1 = min(r0 + share, rows);
    const uint4* qs = reinterpret_cast<const uint4*>(a.q + t * a.q_stride) + c;
    const uint4* ks = reinterpret_cast<const uint4*>(a.k + t * a.k_stride) + c;
    const uint4* vs = reinterpret_cast<const uint4*>(a.v + t * a.v_stride) + c;
    float4 turn[4];
    long long at = -1;                                 // APPEND: the token's slot in kv head 0, in 16-byte vectors; -1: outside the pool
    for (int row0 = r0 + rl; __any_sync(0xffffffffu, row0 < r1); row0 += U * RP) {
        uint4 lo[U], hi[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = row0 + u * RP;
            if (row >= r1) continue;
            const uint4* src = row < nq ? qs + row * (D / 8) : row < nq + nk ? ks + (row - nq) * (D / 8) : vs + (row - nq - nk) * (D / 8);
            lo[u] = __ldcs(src);
            hi[u] = __ldcs(src + TPR);
        }
        if (row0 - rl == r0) {                         // (with the first rows on their way)
            if (a.n_axes) {
#pragma unroll
                for (int x = 0; x < AP; ++x) {
                    double turns = (double)a.positions[(long long)axis[x] * a.T + t] * freq[x];
                    turns -= rint(turns);
                    float s_, c_;
                    sincospif(2.f * (float)turns, &s_, &c_);
                    // frequency j is the (j % 8)-th of lane j / 8 of a row: vector (j % 8) / 2 of that lane, its half j % 2
                    const int j = lane + 32 * x;
                    reinterpret_cast<float2*>(&cs[warp][j % 8 / 2 * TPR + j / 8])[j & 1] = make_float2(c_, s_);
                }
                __syncwarp();
#pragma unroll
                for (int x = 0; x < 4; ++x) turn[x] = cs[warp][x * TPR + c];
            }
            if constexpr (APPEND) {
                int l = 0, r = a.B;                                       // first sequence that ends behind t
                while (l < r) { const int m = (l + r) >> 1; if (cu[m + 1] <= t) l = m + 1; else r = m; }
                if (l >= a.B || t < cu[l]) return;                        // behind the last sequence, or ahead of the first
                const int S = cu[a.B + 1 + l];
                if (S < 0 || S > a.S_max - (cu[l + 1] - cu[l])) return;   // (reported above)
                at = map.at(l, 0, S + (int)t - cu[l], a.Hkv, a.S_max, D / 8);
                if (at < 0 && lane == 0) record_status(a.status, VISPEC_E_RANGE);    // table entry outside the pool: k and v are dropped
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = row0 + u * RP;
            if (row >= r1) continue;
            uint4* dst;
            if (row < nq) {
                dst = reinterpret_cast<uint4*>(a.q_out + t * a.q_out_stride) + row * (D / 8);
            } else if constexpr (APPEND) {
                if (at < 0) continue;
                const bool is_k = row < nq + nk;
                const size_t head = (size_t)(!map.table ? a.S_max : map.token_major ? 1 : map.page_rows) * (D / 8);   // vectors between kv heads
                dst = reinterpret_cast<uint4*>(is_k ? a.k_out : a.v_out) + at + (size_t)(row - nq - (is_k ? 0 : nk)) * head;
            } else {
                dst = reinterpret_cast<uint4*>(a.k_out + t * a.k_out_stride) + (row - nq) * (D / 8);
            }
            if (a.n_axes && row < nq + nk) rotate8(lo[u], hi[u], turn);
            dst[c] = lo[u];
            dst[c + TPR] = hi[u];
        }
    }
}

}  // namespace

cudaError_t launch_prompt_rows(const RowsArgs& a, bool append, int D, int sm_count, cudaStream_t st, const int32_t* block_table,
                               int table_stride, int page_rows, int num_blocks, int token_major) {
    const int rows = (a.q ? a.Hq : 0) + (a.k ? a.Hkv : 0) + (append ? a.Hkv : 0), at_once = 32 / (D / 16);
    if (a.T == 0 && !append) return cudaSuccess;
    // A token's rows are shared out while the SMs have room for more warps, down to the rows that a warp takes at a time.
    const int chunks = std::max(1, std::min((rows + at_once - 1) / at_once, kWarpsPerSm * sm_count / std::max(a.T, 1)));
    const long long items = (long long)std::max(a.T, 1) * chunks;
    const RowMap map = {block_table, table_stride, page_rows, num_blocks, token_major};
    const size_t smem = append ? (size_t)(2 * a.B + 1) * 4 : 0;
    auto go = [&](auto kernel) {
        return launch_pdl(kernel, dim3((unsigned)((items + kRowWarps - 1) / kRowWarps)), dim3(32 * kRowWarps), smem, st, 0, a, map, chunks);
    };
    if (D == 128) return append ? go(prompt_rows_kernel<128, true>) : go(prompt_rows_kernel<128, false>);
    return append ? go(prompt_rows_kernel<64, true>) : go(prompt_rows_kernel<64, false>);
}

}  // namespace vispec
