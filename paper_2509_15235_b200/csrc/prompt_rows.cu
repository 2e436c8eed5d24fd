// Rotary embedding of packed q and k rows by one to four position axes (Sec. 3.2: the target LLM is unchanged; Qwen2.5-VL rotates
// the tokens of an image or a video by time, height and width), alone or on the way of a prompt's rows into the cache.
//
//   x'[j] = x[j] cos a - x[j + D/2] sin a,   x'[j + D/2] = x[j + D/2] cos a + x[j] sin a,   a = positions[axis(j)][t] * theta^(-2j/D)
//
// What bounds it: HBM, every row read once and written once; few rows: the chain launch -> positions -> rotation -> store.  So a
// block forms the D/2 angles of its tokens once and turns all their heads by them, and a thread's first rows are on their way while
// it does so.  An angle is taken as a number of turns, position times frequency / 2 pi in fp64, whose whole part goes before the
// rest (half a turn at most) is rounded to fp32: 2^-26 of a turn, the fp64 part less than that up to positions of 2^22; then
// sine and cosine in fp32, and the products in fp32 with one rounding to bf16.  (Sines in fp64 cost two FP64 warps 400 cycles a
// token, as much as HBM needs for the 20 rows of a 16/2-head model's token.)
#include <cuda_bf16.h>

#include "launch.cuh"
#include "rows.cuh"
#include "vispec_internal.h"

namespace vispec {

namespace {

constexpr int kRowThreads = 256;
constexpr int kTokens = 4;                 // tokens of a block's step at most

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

__device__ __forceinline__ void rotate8(uint4& lo, uint4& hi, const float2* cs) {
    __nv_bfloat162* x = reinterpret_cast<__nv_bfloat162*>(&lo);
    __nv_bfloat162* y = reinterpret_cast<__nv_bfloat162*>(&hi);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const float4 c = *reinterpret_cast<const float4*>(cs + 2 * t);   // (cos, sin) of two frequencies
        const float2 u = __bfloat1622float2(x[t]), w = __bfloat1622float2(y[t]);
        x[t] = __floats2bfloat162_rn(u.x * c.x - w.x * c.y, u.y * c.z - w.y * c.w);
        y[t] = __floats2bfloat162_rn(w.x * c.x + u.x * c.y, w.y * c.z + u.y * c.w);
    }
}

// Rows of a token: Hq of q (if any), Hkv of k (if any), Hkv of v (APPEND).  D/16 threads share a row, each with 8 elements of the
// lower half and the 8 they pair with.  grid.y blocks share a token's rows; grid.x blocks walk the tokens, `tokens` at a time.
template <int D, bool APPEND>
__global__ void __launch_bounds__(kRowThreads)
prompt_rows_kernel(const RowsArgs a, const RowMap map, const int tokens) {
    constexpr int HALF = D / 2, TPR = D / 16, U = 4;
    __shared__ __align__(16) float2 cs[2][kTokens][HALF];
    __shared__ int where_b[2][kTokens], where_slot[2][kTokens];          // APPEND: sequence (-1: the token is left alone) and slot
    extern __shared__ int cu[];                                          // APPEND: B + 1 ends of the sequences
    const int tid = threadIdx.x, aj = tid % HALF, at = tid / HALF;
    const double freq = exp2(-2.0 * (double)aj / (double)D * a.log2_theta) * 0.15915494309189533577;   // turns per position
    const int axis = a.n_axes ? axis_of(aj, a) : 0;
    pdl_wait();
    if constexpr (!APPEND) pdl_launch_dependents();    // (an append writes committed slots: what follows starts when it has ended)
    bool sound = true;
    if constexpr (APPEND) {
        for (int i = tid; i <= a.B; i += kRowThreads) cu[i] = a.cu_len[i];
        __syncthreads();
        for (int i = tid; i < a.B; i += kRowThreads) sound &= cu[i] <= cu[i + 1];
        sound &= cu[0] >= 0 && cu[a.B] <= a.T;
        sound = __syncthreads_and(sound);
        const bool first = blockIdx.x == 0 && blockIdx.y == 0;
        if (!sound) {
            if (first && tid == 0) record_status(a.status, VISPEC_E_RANGE);
            return;
        }
        if (first)
            for (int b = tid; b < a.B; b += kRowThreads) {
                const int S = a.kv_len[b], n = cu[b + 1] - cu[b];
                if (S < 0 || S > a.S_max - n) record_status(a.status, VISPEC_E_RANGE);
                else if (a.kv_len_out) a.kv_len_out[b] = S + n;
            }
    }
    const int nq = a.q ? a.Hq : 0, nk = a.k ? a.Hkv : 0, rows = nq + nk + (APPEND ? a.Hkv : 0);
    const int share = (rows + (int)gridDim.y - 1) / (int)gridDim.y, r0 = blockIdx.y * share, nr = min(share, rows - r0);
    if (nr <= 0) return;
    int buf = 0;
    for (long long t0 = (long long)blockIdx.x * tokens; t0 < a.T; t0 += (long long)gridDim.x * tokens, buf ^= 1) {
        const int nt = (int)min((long long)tokens, a.T - t0), items = nt * nr * TPR;
        for (int base = 0; base < items; base += kRowThreads * U) {
            uint4 lo[U], hi[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int it = base + u * kRowThreads + tid;
                if (it >= items) continue;
                const int ri = it / TPR, c8 = it % TPR * 8, tk = ri / nr, row = r0 + ri - tk * nr;
                const long long t = t0 + tk;
                const __nv_bfloat16* src = row < nq ? a.q + t * a.q_stride + row * D
                                         : row < nq + nk ? a.k + t * a.k_stride + (row - nq) * D
                                                         : a.v + t * a.v_stride + (row - nq - nk) * D;
                lo[u] = __ldcs(reinterpret_cast<const uint4*>(src + c8));
                hi[u] = __ldcs(reinterpret_cast<const uint4*>(src + c8 + HALF));
            }
            if (base == 0) {
                if (a.n_axes && at < nt) {
                    double turns = (double)a.positions[(long long)axis * a.T + t0 + at] * freq;
                    turns -= rint(turns);
                    float s_, c_;
                    sincospif(2.f * (float)turns, &s_, &c_);
                    cs[buf][at][aj] = make_float2(c_, s_);
                }
                if constexpr (APPEND) {
                    if (tid < nt) {
                        const int t = (int)t0 + tid;
                        int l = 0, r = a.B;                               // first sequence that ends behind t
                        while (l < r) { const int m = (l + r) >> 1; if (cu[m + 1] <= t) l = m + 1; else r = m; }
                        int b = -1, slot = 0;
                        if (l < a.B && t >= cu[l]) {
                            const int S = a.kv_len[l];
                            if (S >= 0 && S <= a.S_max - (cu[l + 1] - cu[l])) { b = l; slot = S + t - cu[l]; }
                        }
                        where_b[buf][tid] = b;
                        where_slot[buf][tid] = slot;
                    }
                }
                __syncthreads();
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int it = base + u * kRowThreads + tid;
                if (it >= items) continue;
                const int ri = it / TPR, c8 = it % TPR * 8, tk = ri / nr, row = r0 + ri - tk * nr;
                const long long t = t0 + tk;
                __nv_bfloat16* dst;
                if (APPEND && where_b[buf][tk] < 0) continue;
                if (row < nq) {
                    dst = a.q_out + t * a.q_out_stride + row * D;
                } else if constexpr (APPEND) {
                    const bool is_k = row < nq + nk;
                    const int h = row - nq - (is_k ? 0 : nk);
                    const long long o = map.at(where_b[buf][tk], h, where_slot[buf][tk], a.Hkv, a.S_max, D / 8);
                    if (o < 0) {                                          // table entry outside the pool: the row is dropped
                        if (c8 == 0) record_status(a.status, VISPEC_E_RANGE);
                        continue;
                    }
                    dst = (is_k ? a.k_out : a.v_out) + o * 8;
                } else {
                    dst = a.k_out + t * a.k_out_stride + (row - nq) * D;
                }
                if (a.n_axes && row < nq + nk) rotate8(lo[u], hi[u], &cs[buf][tk][c8]);
                *reinterpret_cast<uint4*>(dst + c8) = lo[u];
                *reinterpret_cast<uint4*>(dst + c8 + HALF) = hi[u];
            }
        }
    }
}

}  // namespace

cudaError_t launch_prompt_rows(const RowsArgs& a, bool append, int D, int sm_count, cudaStream_t st, const int32_t* block_table,
                               int table_stride, int page_rows, int num_blocks, int token_major) {
    const int rows = (a.q ? a.Hq : 0) + (a.k ? a.Hkv : 0) + (append ? a.Hkv : 0), per_pass = kRowThreads / (D / 16);
    if (a.T == 0 && !append) return cudaSuccess;
    // Few tokens: a block per token and pass of rows, so that a thread has one load round trip.  Many: four tokens a step, all rows of
    // a token in one block, blocks that stay.
    const int passes = (rows + per_pass - 1) / per_pass;
    const bool few = (long long)a.T * passes <= 8ll * sm_count;
    const int tokens = few ? 1 : kTokens, gx = few ? (a.T > 0 ? a.T : 1) : min((a.T + kTokens - 1) / kTokens, 6 * sm_count), gy = few ? passes : 1;
    const RowMap map = {block_table, table_stride, page_rows, num_blocks, token_major};
    const size_t smem = append ? (size_t)(a.B + 1) * 4 : 0;
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(gx, gy), dim3(kRowThreads), smem, st, 0, a, map, tokens); };
    if (D == 128) return append ? go(prompt_rows_kernel<128, true>) : go(prompt_rows_kernel<128, false>);
    return append ? go(prompt_rows_kernel<64, true>) : go(prompt_rows_kernel<64, false>);
}

}  // namespace vispec
