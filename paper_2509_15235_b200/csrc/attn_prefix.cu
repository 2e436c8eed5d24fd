// Attention of a batch whose sequences share a long prefix (several samples, questions or drafts behind one image or video), on a
// paged cache whose block tables start with the same blocks: the prefix is read once and scored against the query rows of all
// sequences together, and each sequence's own keys against its own rows.
//
//   For a query row: (m_p, l_p, o_p) over each piece p of its keys, m_p the reference maximum (log2 units), l_p = sum 2^(s - m_p),
//   o_p = sum 2^(s - m_p) v;   m = max m_p,  l = sum l_p 2^(m_p - m),  out = sum o_p 2^(m_p - m) / l,  lse = (m + log2 l) ln 2.
//
// What bounds it: trees of a few sequences make hundreds of rows per kv head, and the prefix costs 4 D flops for each of them a key, so
// the tensor pipe and the exponentials bound it; with one row per sequence (single-token decoding) it is the read of the keys.
//
// Work.  Two kinds of units: (kv head, block of 256 of the batch's B*N*G rows) over the prefix, and (sequence, kv head, block of 256
// of its N*G rows) over its own keys, both in steps of 128 keys.  All steps lie on one line, the prefix units first, each with its
// cost (a unit's start costs too), and every CTA, one per SM, takes an equal range of it: no case needs a choice of how many SMs
// the prefix gets, and kv_len, which the device alone knows, decides.  A CTA's part of a unit is a segment; each segment parks its rows' (m, l, o)
// in the scratch, and a second kernel adds up a row's pieces.  (A prefix unit and a sequence's unit always have two pieces to
// add, so there is nothing to gain from finishing a row in the first kernel.)  With few rows per sequence and kv head, the sequences'
// own keys are few_rows_kernel's (below), which also joins the pieces, and the prefix is alone on the line.  That, and what goes with it (the cut
// of the prefix's units, warps and clusters per unit), the host chooses, by the lengths that it has to expect (own_keys).
//
// Measured, us of a call among others with changing inputs (floor: bytes at 6516 GB/s or flops at 1652 TFLOP/s):
//   8 x 128 nodes of 16/2 heads on 32768 shared + 300 to 2048 own keys    275 (173, tensor): 1.04 PFLOP/s
//   8 x 60 nodes of 32/32 heads on 3904 + 46 to 354                        66 (19.8, tensor)
//   4 x 60 nodes of 28/4 heads on 3344 + 46 to 354                         27.1 (7.5, tensor)
//   32 x 1 node of 40/40 heads on 2880 + 46 to 354                         55.7 (29.4, HBM), few rows
//   8 x 1 node of 28/4 heads on 3344 + 46 to 354                           14.9 (1.6, HBM), few rows: two dependent launches
//
// A segment runs on two accumulator tiles of 128 rows, each with four softmax warps, one thread per row, which work out of phase so that
// the tensor pipe serves one while the other is in its exponentials, as in attn_tc5_wide.cu:
//   wide        more than 128 rows: the tiles hold different rows and share every K/V stage
//   alternate   at most 128 rows: both tiles hold the same rows and take turns at the steps; a row has two parts
// In terms of "operations" 0, 1, 2, ... (one tile's share of a step; the tiles take turns, across segments too) the issue order is
// always S(0) S(1) | PV(0) S(2) | PV(1) S(3) | ...
//
//   warp 0  producer of the K ring (2 x 32 KB)      warp 2  producer of the V ring (3 x 32 KB)
//   warp 1  issuer of all products                   warp 3  derives the schedule from kv_len, then fetches alternate segments' Q rows
//   warps 4-7 / 8-11  softmax of tile A / B: thread <-> TMEM lane <-> query row
// TMEM (512 columns): S_A 0..127, S_B 128..255 (P of the tile, bf16, in the first 64 columns of its S), O_A 256, O_B 384.
// The waits, time-outs and the programmatic launch are those of attn_tc5.cu.
#include <cuda_bf16.h>
#include <algorithm>

#include "tc5_common.cuh"

namespace vispec {

using namespace tc5;

namespace {

constexpr int kThreads = 384;
constexpr int kRows = 256;                     // query rows of a unit
constexpr int kMaxLineB = 64;                  // sequences whose own keys are on the line (few_rows_kernel takes any number)
constexpr uint32_t TMEM_COLS = 512;
constexpr uint32_t COL_S = 0, COL_O = 256;     // + 128 per tile

enum { X_KFULL = 0, X_KEMPTY = X_KFULL + 2, X_VFULL = X_KEMPTY + 2, X_VEMPTY = X_VFULL + 3, X_SFULL = X_VEMPTY + 3,
       X_PFULL = X_SFULL + 2 /* [tile][half of the columns] */, X_QWIDE = X_PFULL + 4, X_QALT = X_QWIDE + 2, X_QEMPTY = X_QALT + 2,
       X_OFULL = X_QEMPTY + 2, X_OFREE = X_OFULL + 2, X_STAT = X_OFREE + 2, X_COUNT = X_STAT + 1 };

struct PrefixRing {
    static constexpr int STAGE = 2 * HALF_BYTES, NSK = 2, NSV = 3;
    static constexpr int OFF_K = 0, OFF_V = NSK * STAGE, OFF_Q = OFF_V + NSV * STAGE;
    static constexpr int KFULL = X_KFULL, KEMPTY = X_KEMPTY, VFULL = X_VFULL, VEMPTY = X_VEMPTY;
};
constexpr int SMEM_BAR = 7 * PrefixRing::STAGE;
constexpr int BAR_BYTES = 240;
static_assert(X_COUNT * 8 + 20 <= BAR_BYTES, "barrier block too small");
constexpr int SMEM_SCHED = SMEM_BAR + BAR_BYTES;

// Where things lie on the line.  Group 0 is the prefix, group b + 1 sequence b.
struct PrefixSched {
    int base[kMaxLineB + 2];       // where group g starts; base[groups + 1] = length of the line
    int len[kMaxLineB];            // sequence b's own committed slots; -1: rejected
    int range;                     // places of the line per CTA
};
constexpr int SMEM_TABRING = SMEM_SCHED + ((int)sizeof(PrefixSched) + 15) / 16 * 16;
constexpr int SMEM_STAT = SMEM_TABRING + 256;   // (m, l) of both tiles' rows, exchanged at the end of an alternate segment
constexpr int SMEM_ALLOC = SMEM_STAT + 256 * 8;
static_assert(SMEM_ALLOC <= 232448, "over the 227 KB a CTA may have");

struct PrefixParams {
    const __nv_bfloat16* q; const int32_t* kv_len; const uint64_t* mask;
    __nv_bfloat16* out; float* lse;
    // partials: slot s of a region is [D/4][slot_rows] float4 and [slot_rows] (m, l): the unit's rows, or where an alternate segment's
    // parts are two pieces, the second one half the slot behind the first
    float4* part_o[2]; float2* part_ml[2];     // [0] prefix units, [1] sequences' own
    int slot_rows[2], blocks[2], last_alt[2];  // rows of a slot; row blocks per kv head; is the last one alternate?
    int B, N, Hq, Hkv, G;
    int P, cap;                                // keys of the prefix; slots a sequence may have beyond it
    int early, grid;
    int pad, range;                            // prefix alone on a line shorter than the SMs: places of a unit, and of a CTA (0: see range_of)
    int groups;                                // sequences whose own keys are on the line: B, or 0 where few_rows_kernel takes them
    float scale_log2;
    int* status;
};

// Places of the line (some 210 cycles each, from clock stamps of 8 x 60 nodes of 32/32 heads): a wide step 3400 cycles, an alternate
// one 1900, the start of a segment (Q rows, first score, last product, partials) 7500 and 3500.
// (Starts of 16 to 36 and 10 to 24 places, alternate steps of 8 to 12: within 5 % of one another on nine shapes, these the best for the
// longest.)  A range of fewer than kMinRange places costs more to start and to join than it saves: 26 to 36 the same, 44 and 48 6 % more
// on 8 single tokens of 28/4 heads.
constexpr int kWideStep = 16, kAltStep = 9, kWideStart = 36, kAltStart = 16, kMinRange = 32;
__host__ __device__ constexpr int step_places(bool alt) { return alt ? kAltStep : kWideStep; }
__host__ __device__ constexpr int start_places(bool alt) { return alt ? kAltStart : kWideStart; }

__host__ __device__ __forceinline__ int unit_places(const PrefixParams& p, int kind, int steps, bool last) {
    if (kind == 0 && p.pad) return p.pad;
    const bool alt = last && p.last_alt[kind];
    return start_places(alt) + steps * step_places(alt);
}
__host__ __device__ __forceinline__ int head_places(const PrefixParams& p, int kind, int steps) {
    return steps == 0 ? 0 : (p.blocks[kind] - 1) * unit_places(p, kind, steps, false) + unit_places(p, kind, steps, true);
}
__device__ __forceinline__ int own_len(const PrefixParams& p, int kv) {       // -1: rejected
    return kv >= p.P && kv - p.P <= p.cap - p.N ? kv - p.P : -1;
}
__host__ __device__ __forceinline__ int steps_of(int keys) { return (keys + STEP - 1) / STEP; }

// One warp: exclusive sums of the sequences' places behind the prefix, and the range of a CTA.  store(b, base, len) for each sequence.
template <typename F>
__device__ __forceinline__ int line_build(const PrefixParams& p, int lane, const int* kv, F&& store) {
    int carry = p.Hkv * head_places(p, 0, steps_of(p.P));
#pragma unroll
    for (int i = 0; i < kMaxLineB / 32; ++i) {
        if (i * 32 >= p.groups) break;
        const int b = i * 32 + lane;
        const int S = b < p.groups ? own_len(p, kv[i]) : -1;
        const int len = S >= 0 ? p.Hkv * head_places(p, 1, steps_of(S + p.N)) : 0;
        int x = len;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        store(i, b, carry + x - len, S);
        carry += __shfl_sync(0xffffffffu, x, 31);
    }
    return carry;
}
__host__ __device__ __forceinline__ int range_of(const PrefixParams& p, int T) {
    const int even = (T + p.grid - 1) / p.grid;
    return p.range ? p.range : even > kMinRange ? even : kMinRange;
}

// The first step of a unit that starts at `start` whose place is at or behind g.
__device__ __forceinline__ int step_at(int g, int start, bool alt) {
    const int d = g - start - start_places(alt);
    return d <= 0 ? 0 : alt ? (d + kAltStep - 1) / kAltStep : (d + kWideStep - 1) / kWideStep;
}

struct PSeg {
    int b;                    // sequence; 0 for the prefix (its row of the block table is the one that is read)
    int kind, kvh, st0, n;    // 0 prefix, 1 own keys; kv head; first step and their number
    int S, total;             // committed keys of the unit, all keys (with the tree's rows)
    int node0, rows0, rows;   // q row r (of `rows`) of the unit is head (rows0 + r) % G of node node0 + (rows0 + r) / G
    int slot;
    bool alt;
};

// A CTA's segments, in their order.  Only the first unit is looked up; from one unit to the next it goes by counting (a lookup's
// divisions and dependent loads took every role 1500 cycles a segment, a sixth of a short segment).
struct PIter {
    const PrefixSched* s; const PrefixParams* p;
    int lo, hi, cta;
    int grp, kvh, m, start;                  // the unit that comes next: group, kv head, row block, where it starts
    int kind, steps, full, last;             // its group: prefix or own, steps of a unit, places of one with 256 rows, of a head's last one
    __device__ __forceinline__ void enter() {
        kind = grp > 0 ? 1 : 0;
        steps = steps_of(kind ? s->len[grp - 1] + p->N : p->P);
        full = unit_places(*p, kind, steps, false);
        last = unit_places(*p, kind, steps, true);
    }
    __device__ __forceinline__ PIter(const PrefixSched* s_, const PrefixParams* p_, int lo_, int hi_, int cta_)
        : s(s_), p(p_), lo(lo_), hi(hi_), cta(cta_), grp(0), kvh(0), m(0), start(hi_) {
        if (lo >= hi) return;
        int l = 0, r = p->groups + 1;                                    // first group with base > lo, minus one
        while (l < r) { const int x = (l + r) >> 1; if (s->base[x] <= lo) l = x + 1; else r = x; }
        grp = l - 1;
        enter();
        const int rel = lo - s->base[grp], head = (p->blocks[kind] - 1) * full + last;
        kvh = rel / head;
        m = min((rel - kvh * head) / full, p->blocks[kind] - 1);
        start = s->base[grp] + kvh * head + m * full;
    }
    __device__ __forceinline__ bool next(PSeg& o) {
        while (start < hi) {
            const int nb = p->blocks[kind], here = start;
            o.kind = kind;
            o.b = kind ? grp - 1 : 0;
            o.S = kind ? s->len[grp - 1] : p->P;
            o.total = kind ? o.S + p->N : o.S;
            o.kvh = kvh;
            o.rows0 = m * kRows;
            o.rows = min(kRows, (kind ? p->N : p->B * p->N) * p->G - o.rows0);
            o.alt = o.rows <= 128;
            o.node0 = o.b * p->N;
            o.slot = (o.b * p->Hkv + kvh) * nb + m + cta;           // units and CTAs both only go up along the line
            o.st0 = 0;
            o.n = steps;
            start += m == nb - 1 ? last : full;
            if (here < lo) o.st0 = step_at(lo, here, o.alt);
            if (start > hi) o.n = min(steps, step_at(hi, here, o.alt));     // (a padded unit ends behind its last step)
            o.n -= o.st0;
            if (++m == nb) {
                m = 0;
                if (++kvh == p->Hkv) {
                    kvh = 0;
                    do ++grp; while (grp <= p->groups && s->base[grp + 1] == start);     // groups without units
                    if (start < hi) enter();
                }
            }
            if (o.n > 0) return true;
        }
        return false;
    }
};

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// (pa is not __grid_constant__: the producers hand a changed copy of it on, and with the attribute nvcc 12.9 passed the original)
// ALONE: no sequence's own keys are on the line.  Then the two parts of a row that an alternate segment has are added up at its end,
// because few_rows_kernel reads them for every sequence anew; otherwise they are two pieces (adding them up makes each tile wait for
// the other, which costs the short segments of the sequences' own keys more than the pieces do: 60.9 -> 66.0 us for 8 trees of 60 nodes
// of 32/32 heads, against 49.8 -> 46.5 us for 32 single tokens of 40/40 heads).
template <bool ALONE>
__global__ void __launch_bounds__(kThreads, 1)
attn_prefix_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map, const __grid_constant__ PrefixParams p,
                   const PagedArgs pa) {
    using R = PrefixRing;
    constexpr int NSK = R::NSK, NSV = R::NSV, STAGE = R::STAGE;
    extern __shared__ __align__(1024) unsigned char sm[];
    const uint32_t base = smem_u32(sm);
    if (base & 1023u) {                        // the swizzled tiles need it; every CTA sees the same base, so all of them leave
        if (threadIdx.x == 0) atomicCAS(p.status, 0, (int)VISPEC_E_UNSUPPORTED);
        return;
    }
    const uint32_t bars = base + SMEM_BAR;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sm + SMEM_BAR + X_COUNT * 8);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(sm + SMEM_BAR + X_COUNT * 8 + 8);
    PrefixSched& sched = *reinterpret_cast<PrefixSched*>(sm + SMEM_SCHED);
    auto bar = [&](int i) { return bars + 8u * (uint32_t)i; };
    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    const int cta = blockIdx.x;

    if (tid == 0) {
        for (int i = 0; i < NSK; ++i) { mbar_init(bar(X_KFULL + i), 1); mbar_init(bar(X_KEMPTY + i), 1); }
        for (int i = 0; i < NSV; ++i) { mbar_init(bar(X_VFULL + i), 1); mbar_init(bar(X_VEMPTY + i), 1); }
        for (int i = 0; i < 4; ++i) mbar_init(bar(X_PFULL + i), 128);
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar(X_SFULL + i), 1);
            mbar_init(bar(X_QWIDE + i), 129); mbar_init(bar(X_QALT + i), 32); mbar_init(bar(X_QEMPTY + i), 1);
            mbar_init(bar(X_OFULL + i), 1); mbar_init(bar(X_OFREE + i), 128);
        }
        mbar_init(bar(X_STAT), 256);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (!p.early) pdl_wait();
    if (warp == 3) {
        int kv[kMaxLineB / 32];
#pragma unroll
        for (int i = 0; i < kMaxLineB / 32; ++i) kv[i] = i * 32 + lane < p.groups ? p.kv_len[i * 32 + lane] : 0;
        const int T = line_build(p, lane, kv, [&](int, int b, int at, int S) {
            if (b < p.groups) { sched.base[b + 1] = at; sched.len[b] = S; }
        });
        if (lane == 0) { sched.base[0] = 0; sched.base[p.groups + 1] = T; sched.range = range_of(p, T); }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto make_iter = [&]() {
        const int T = sched.base[p.groups + 1], lo = (int)min((long long)cta * sched.range, (long long)T);
        return PIter(&sched, &p, lo, min(lo + sched.range, T), cta);
    };

    if (warp == 0 || warp == 2) {
        // ================= TMA producers: warp 0 the K ring, warp 2 the V ring =================
        const bool is_v = warp == 2;
        const uint64_t once = l2_evict_first_policy(), again = l2_evict_normal_policy();
        bool waited = !p.early, ok = true;
        int it = 0;
        PIter si = make_iter();
        PSeg sg;
        const int ns = is_v ? NSV : NSK, full = is_v ? X_VFULL : X_KFULL;
        while (ok && si.next(sg)) {
            PagedArgs a = pa;
            a.N = sg.total - sg.S;
            if (sg.kind) a.block_table += p.P / pa.page_rows;
            const uint32_t r = produce_paged<R>(a, &k_map, &v_map, sg.b, sg.kvh, sg.st0, sg.n, sg.S, base, bars,
                                                base + SMEM_TABRING + (is_v ? 128 : 0), abort_flag, p.blocks[sg.kind] > 1 ? again : once, it, waited, lane, is_v ? 2 : 1);
            it += (int)(r & 0x0fffffffu) + (is_v ? 0 : (int)((r >> 28) & 1u));
            ok = !((r >> 29) & 1u);
            waited = (r >> 30) & 1u;
        }
        if (*abort_flag && lane == 0) {
            // drain: wait (bounded, fresh timer) until every copy this warp issued has landed
            volatile int never = 0;
            for (int u = max(0, it - ns); u < it; ++u) mbar_wait(bar(full + u % ns), (u / ns) & 1, &never);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ================= issuer of all products (one elected lane; the whole warp walks and waits) =================
        constexpr uint32_t IDESC_S = instr_desc(0), IDESC_O = instr_desc(1, D);
        constexpr uint32_t DESC_HI = desc_hi(1024);
        const bool leader = elect_one();
        const uint32_t k0 = desc_lo(base + R::OFF_K, 16), v0 = desc_lo(base + R::OFF_V, HALF_BYTES), q0 = desc_lo(base + R::OFF_Q, 16);
        PIter si = make_iter();
        PSeg sg;
        uint32_t sk = 0, pk = 0, sv = 0, pv = 0, pp = 0;   // ring positions with their phases; bit x of pp: phase of tile x's P
        uint32_t qw = 0, qa = 0, qr = 0;                   // phases of the Q barriers: wide segments, bit r: region r; next region
        int sx = 0, px = 0, seg = 0;                       // alternate segments: tiles of the next score and PV product
        bool ok = true;
        // this segment and the one behind it: 0 steps where there is none
        auto fetch = [&](int& n, bool& alt) {
            const bool live = si.next(sg);
            alt = __shfl_sync(0xffffffffu, (int)sg.alt, 0) != 0;
            n = live ? __shfl_sync(0xffffffffu, sg.n, 0) : 0;
        };
        auto wait = [&](int i, uint32_t parity) { return ok = mbar_wait_warp(bar(i), parity, abort_flag); };
        // S_x = Q K^T of the K stage sk, Q from region r
        auto score = [&](int x, uint32_t r, bool stage_done, bool q_done) {
            tc_fence_after();
            if (leader) {
                const uint32_t kb = k0 + sk * (STAGE >> 4), qb = q0 + r * (STAGE >> 4);
#pragma unroll
                for (int ks = 0; ks < D / 16; ++ks) {
                    const uint32_t off = ((ks >> 2) * HALF_BYTES + (ks & 3) * 32) >> 4;
                    tc_mma_ss(tmem + COL_S + x * 128, qb + off, DESC_HI, kb + off, DESC_HI, IDESC_S, ks > 0 ? 1u : 0u);
                }
                tc_commit(bar(X_SFULL + x));
                if (stage_done) tc_commit(bar(X_KEMPTY) + 8u * sk);
                if (q_done) tc_commit(bar(X_QEMPTY) + 8u * r);                     // the last score from this Q region
            }
            if (stage_done && ++sk == NSK) { sk = 0; pk ^= 1; }
        };
        // O_x (+)= P_x V of the V stage sv, half of the tokens as soon as their P is there
        auto product = [&](int x, bool fresh, bool stage_done) {
            const uint32_t vb = v0 + sv * (STAGE >> 4);
            // (a segment's first PV product starts a fresh O: the last segment's must have been read)
            if (!ALONE && fresh && seg > 0 && !wait(X_OFREE + x, (seg - 1) & 1)) return;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!wait(X_PFULL + 2 * x + h, (pp >> x) & 1)) return;
                tc_fence_after();
                if (leader) {
#pragma unroll
                    for (int ks = h * (STEP / 32); ks < (h + 1) * (STEP / 32); ++ks)
                        tc_mma_ts(tmem + COL_O + x * 128, tmem + COL_S + x * 128 + ks * 8, vb + ks * 128, DESC_HI, IDESC_O, (!fresh || ks > 0) ? 1u : 0u);
                }
            }
            pp ^= 1u << x;
            if (stage_done) {
                if (leader) tc_commit(bar(X_VEMPTY) + 8u * sv);
                if (++sv == NSV) { sv = 0; pv ^= 1; }
            }
        };
        // (ALONE: by both tiles' threads, where it was an alternate segment)
        auto o_free = [&]() { return !ALONE || seg == 0 || (wait(X_OFREE, (seg - 1) & 1) && wait(X_OFREE + 1, (seg - 1) & 1)); };
        // An alternate segment's next score, if it may be issued (wait_for_it: as soon as it may).
        auto alt_score = [&](int j, int n, bool wait_for_it) {
            auto have = [&](int i, uint32_t parity) {
                return wait_for_it ? wait(i, parity) : __all_sync(0xffffffffu, mbar_test(bar(i), parity)) != 0;
            };
            if ((j == 0 && !have(X_QALT + (int)qr, (qa >> qr) & 1)) || !have(X_KFULL + (int)sk, pk)) return 0;
            score(sx, qr, true, j + 1 == n);
            if (j + 1 == n) { qa ^= 1u << qr; qr ^= 1; }
            sx ^= 1;
            return 1;
        };
        int n, n1, scored = 0;                             // steps of this segment and of the next, scores of this one issued so far
        bool alt, alt1;
        fetch(n, alt);
        while (ok && n > 0) {
            int scored1 = 0;
            if (alt) {
                while (ok && scored < 2 && scored < n) scored += alt_score(scored, n, true);
                fetch(n1, alt1);
                for (int j = 0; j < n && ok; ++j) {
                    if (!wait(X_VFULL + (int)sv, pv) || (j == 0 && !o_free())) break;
                    product(px, j < 2, true);
                    if (!ok) break;
                    if (j + 2 >= n && leader) tc_commit(bar(X_OFULL + px));
                    if (n == 1) {
                        // (the tile without an operation keeps step as well: neither side may be two phases ahead of the other)
                        if (!ALONE && seg > 0 && !wait(X_OFREE + (px ^ 1), (seg - 1) & 1)) break;
                        if (leader) tc_commit(bar(X_OFULL + (px ^ 1)));
                    }
                    px ^= 1;
                    // the tile's next score (overwrites P of this operation, which the product before it reads): of this segment, or of
                    // the next one where that is an alternate one (a wide one's Q rows come from threads that first have to end this
                    // segment) and its operands are there already (a wait here would hold up this segment's products)
                    if (scored < n) scored += alt_score(scored, n, true);
                    else if (alt1 && scored1 < n1) scored1 += alt_score(scored1, n1, false);
                }
            } else {
                for (int x = 0; x < 2 && ok; ++x)
                    if (wait(X_QWIDE + x, qw) && (x == 1 || wait(X_KFULL + (int)sk, pk))) score(x, x, x == 1, n == 1);
                qw ^= 1;
                fetch(n1, alt1);
                for (int t = 0; t < n && ok; ++t) {
                    if (!wait(X_VFULL + (int)sv, pv) || (t == 0 && !o_free())) break;
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        if (!ok) break;
                        product(x, t == 0, x == 1);
                        if (!ok) break;
                        if (t + 1 < n) {                   // overwrites P of this step, which the product before it reads
                            if (x == 1 || wait(X_KFULL + (int)sk, pk)) score(x, x, x == 1, t + 2 == n);
                        } else if (leader) {
                            tc_commit(bar(X_OFULL + x));
                        }
                    }
                }
                sx = px = 0;
            }
            ++seg;
            n = n1; alt = alt1; scored = scored1;
        }
        __syncwarp();
    } else if (warp == 3) {
        // ================= Q rows of the alternate segments: both tiles score the same rows, so the two Q regions take turns and the
        // next segment's rows are there before this one has ended (wide segments need both, the softmax threads fill them)
        pdl_wait();
        PIter si = make_iter();
        PSeg sg;
        int fills[2] = {0, 0}, qr = 0;
        bool ok = true;
        while (ok && si.next(sg)) {
            // (every use of a region is waited for in its turn, also those that the softmax threads fill, and is held up until it has
            // been: a parity tells only the last two phases apart)
            if (!sg.alt || qr == 0) ok = mbar_wait_warp(bar(X_QEMPTY), (fills[0]++ & 1) ^ 1, abort_flag);
            if (ok && (!sg.alt || qr == 1)) ok = mbar_wait_warp(bar(X_QEMPTY + 1), (fills[1]++ & 1) ^ 1, abort_flag);
            if (!ok) break;
            if (!sg.alt) {
                if (lane < 2) mbar_arrive(bar(X_QWIDE + lane));
                continue;
            }
            // half a warp per row, one 16-byte chunk a lane, into the swizzled K-major layout of a K stage.  Rows that do not exist keep
            // what is there: a row's scores are its own
            const int c = lane & 15, r0 = lane >> 4;
            const uint32_t dst = base + R::OFF_Q + qr * STAGE + (c >> 3) * HALF_BYTES;
            int nd = sg.node0 + (sg.rows0 + r0) / p.G, g = (sg.rows0 + r0) % p.G;
#pragma unroll 4
            for (int r = r0; r < sg.rows; r += 2) {
                cp_async16(dst + r * 128 + (((c & 7) ^ (r & 7)) << 4), p.q + ((size_t)nd * p.Hq + sg.kvh * p.G + g) * D + c * 8);
                g += 2;
                while (g >= p.G) { g -= p.G; ++nd; }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            fence_async_smem();
            mbar_arrive(bar(X_QALT) + 8u * qr);
            qr ^= 1;
        }
    } else if (warp >= 4) {
        // ================= softmax: one thread per query row, tile x by warps 4 + 4x .. 7 + 4x =================
        const int x = (warp - 4) >> 2, sp = warp & 3;
        const int tl = sp * 32 + lane;                        // TMEM lane = row of the tile
        const uint32_t lane_addr = tmem + ((uint32_t)(32 * sp) << 16);
        const uint32_t s_addr = lane_addr + COL_S + x * 128, o_addr = lane_addr + COL_O + x * 128;
        pdl_wait();                                           // q, tree_mask and every output come after the preceding kernel
        pdl_launch_dependents();                              // (few_rows_kernel, which may follow, reads q ahead of its own wait)
        const int G = p.G, N = p.N;
        PIter si = make_iter();
        PSeg sg;
        int it = 0, steps_before = 0, x0 = 0;                 // operations of this tile so far / steps of all segments so far / tile that begins
        uint32_t o_phase = 0, stat_phase = 0;
        int fills[2] = {0, 0}, qr = 0;                        // how often each Q region has been filled; the next alternate segment's
        bool ok = true;
        // wide: Q tile -> shared memory, rows in the swizzled K-major layout of a K stage, asked for here and handed over by q_here.
        // Thread t moves chunk t % 16 of rows t / 16, t / 16 + 8, ... (a loop of little code: unrolled with its divisions it took 8000
        // cycles, most of them the fetch of its code).  Rows that do not exist keep what is there: a row's scores are its own.
        auto q_ask = [&]() {
            if (sg.alt) {
                if (qr) ++fills[1]; else ++fills[0];
                qr ^= 1;
                return;
            }
            if (!(ok = mbar_wait_warp(bar(X_QEMPTY + x), ((x ? fills[1] : fills[0]) & 1) ^ 1, abort_flag))) return;
            ++fills[0]; ++fills[1];
            const int c = tl & 15, step_nd = 8 / G, step_g = 8 % G, row0 = sg.rows0 + x * 128 + (tl >> 4), end = min(128, sg.rows - x * 128);
            const uint32_t dst = base + R::OFF_Q + x * STAGE + (c >> 3) * HALF_BYTES;
            int nd = sg.node0 + row0 / G, g = row0 % G;
#pragma unroll 2
            for (int r = tl >> 4; r < end; r += 8) {
                cp_async16(dst + r * 128 + (((c & 7) ^ (r & 7)) << 4), p.q + ((size_t)nd * p.Hq + sg.kvh * G + g) * D + c * 8);
                nd += step_nd;
                g += step_g;
                if (g >= G) { g -= G; ++nd; }
            }
        };
        bool live = si.next(sg);
        if (live) q_ask();
        while (ok && live) {
            const int tile0 = sg.alt ? 0 : x * 128;           // this tile's first row in the unit
            if (!sg.alt) {
                asm volatile("cp.async.wait_all;" ::: "memory");
                fence_async_smem();
                mbar_arrive(bar(X_QWIDE + x));
            }
            const bool row_ok = tile0 + tl < sg.rows;
            const bool warp_rows = tile0 + sp * 32 < sg.rows;     // a warp without rows only keeps the barriers going
            const int S = sg.S, total = sg.total;
            uint64_t mk0 = 0, mk1 = 0;
            if (row_ok && sg.kind) {
                const int W = (N + 63) >> 6;
                const uint64_t* mrow = p.mask + ((size_t)sg.node0 + (sg.rows0 + tile0 + tl) / G) * W;
                mk0 = mrow[0];
                if (W > 1) mk1 = mrow[1];
                if (N < 64) mk0 &= (1ull << N) - 1;           // bits at or beyond N are not tree nodes
                if (N < 128) mk1 &= N > 64 ? (1ull << (N - 64)) - 1 : 0ull;
            }
            float m_ref = -INFINITY, l_run = 0.f;
            bool has_o = false;

            for (int t = sg.alt ? x ^ x0 : 0; t < sg.n; t += sg.alt ? 2 : 1, ++it) {
                const int tok0 = (sg.st0 + t) * STEP;
                // (this product was issued after the tile's last PV product, so that one is complete too: O and the columns of P are free)
                if (!mbar_wait_warp(bar(X_SFULL + x), it & 1, abort_flag)) { ok = false; break; }
                tc_fence_after();
                bool fail = false;
                if (tok0 + STEP > total) {
                    // the unit's last step: V rows past the last key may hold anything, and they meet zero weights: made zeros before
                    // the product (wide: both tiles' warps write them, whichever product comes first)
                    const int sv = (steps_before + t) % NSV;
                    fail = !mbar_wait(bar(X_VFULL + sv), ((steps_before + t) / NSV) & 1, abort_flag);
                    if (!fail) {                              // (consecutive threads write consecutive vectors: a row per thread met one bank)
                        unsigned char* v0 = sm + R::OFF_V + sv * STAGE;
                        for (int i = (total - tok0) * 8 + tl; i < STEP * 8; i += 128) {
                            *reinterpret_cast<uint4*>(v0 + i * 16) = make_uint4(0, 0, 0, 0);
                            *reinterpret_cast<uint4*>(v0 + HALF_BYTES + i * 16) = make_uint4(0, 0, 0, 0);
                        }
                    }
                    fence_async_smem();
                }
                if (__any_sync(0xffffffffu, fail)) { ok = false; break; }
                if (!warp_rows) {
                    tc_fence_before();
                    mbar_arrive(bar(X_PFULL + 2 * x));
                    mbar_arrive(bar(X_PFULL + 2 * x + 1));
                    has_o = true;
                    continue;
                }
                if (tok0 + STEP > S) {
                    // reaches past the committed keys: columns that the row must not see become -inf in tensor memory, so that the
                    // passes below know nothing of masks (in each of them, unrolled, a masked step took 2000 cycles more)
                    uint64_t a0, a1;                                // bit c of (a0, a1): column c may be attended to
                    const int t0 = tok0 - S;
                    if (t0 >= 0) shr128(mk0, mk1, t0, a0, a1); else shl128_fill(mk0, mk1, -t0, a0, a1);
#pragma unroll 1
                    for (int c = 0; c < 4; ++c) {
                        const uint64_t a = c & 2 ? a1 : a0;
                        const uint32_t w = (uint32_t)(c & 1 ? a >> 32 : a);
                        if (__all_sync(0xffffffffu, w == 0xffffffffu)) continue;
                        uint32_t v[32];
                        tmem_ld32(s_addr + c * 32, v);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (!((w >> e) & 1u)) v[e] = 0xff800000u;
                        tmem_st32(s_addr + c * 32, v);
                    }
                    tmem_wait_st();
                }
                // The row is read from tensor memory in halves of 64 columns, the upper half twice (see attn_tc5_wide.cu).
                uint32_t s[64];
                auto load_half = [&](int h) {
                    tmem_ld32(s_addr + h * 64, s);
                    tmem_ld32(s_addr + h * 64 + 32, s + 32);
                    tmem_wait_ld();
                };
                float mx[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) mx[e] = -INFINITY;
#pragma unroll 1
                for (int h = 1; h >= 0; --h) {
                    load_half(h);
#pragma unroll
                    for (int c = 0; c < 64; c += 16)
#pragma unroll
                        for (int e = 0; e < 8; ++e) mx[e] = max3_nan(mx[e], __uint_as_float(s[c + e]), __uint_as_float(s[c + 8 + e]));
                }
                const float tmax = max_nan(max3_nan(max3_nan(mx[0], mx[1], mx[2]), max3_nan(mx[3], mx[4], mx[5]), mx[6]), mx[7]) * p.scale_log2;
                // move the reference maximum only when the tile exceeds it by more than the gap
                float alpha = 1.f;
                bool rescale = false;
                if (tmax > m_ref + kRescaleGap) {         // also true on the first finite tile (m_ref = -inf)
                    alpha = exp2f(m_ref - tmax);
                    m_ref = tmax;
                    l_run *= alpha;
                    rescale = has_o;
                }
                if (!(tmax < INFINITY)) l_run = tmax - tmax;          // a NaN or an infinite score: the row is NaN (see inv_sum)
                if (__any_sync(0xffffffffu, rescale)) {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t o[16];
                        tmem_ld16(o_addr + c * 16, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                        tmem_st16(o_addr + c * 16, o);
                    }
                }
                const float m_use = (m_ref == -INFINITY) ? 0.f : m_ref;
                const uint64_t sc2 = pk2(p.scale_log2, p.scale_log2), mm2 = pk2(-m_use, -m_use);
                uint64_t sum2 = pk2(0.f, 0.f), sum2b = sum2;
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    if (h == 1) load_half(1);             // (P of the first half lies in columns 0..31)
                    uint32_t pd[32];
#pragma unroll
                    for (int c = 0; c < 32; ++c) {
                        float x0, x1;
                        up2(fma2(pk2(__uint_as_float(s[2 * c]), __uint_as_float(s[2 * c + 1])), sc2, mm2), x0, x1);
                        const float e0 = exp2f(x0), e1 = exp2f(x1);
                        if (c & 1) sum2b = add2(sum2b, pk2(e0, e1)); else sum2 = add2(sum2, pk2(e0, e1));
                        pd[c] = pack_bf16(e0, e1);
                    }
                    tmem_st32(s_addr + h * 32, pd);
                    tmem_wait_st();
                    tc_fence_before();
                    mbar_arrive(bar(X_PFULL + 2 * x + h));
                }
                float l0, l1;
                up2(add2(sum2, sum2b), l0, l1);
                l_run += l0 + l1;
                has_o = true;
            }
            if (!ok) break;
            steps_before += sg.n;
            const int piece = sg.alt ? x ^ x0 : x;            // (an alternate segment of one step has only the piece of the tile that began)
            x0 = sg.alt ? x0 ^ (sg.n & 1) : 0;

            // ---- segment epilogue: the row's partial; the next segment's Q rows are asked for first ----
            const bool alt = sg.alt;
            const int rows = p.slot_rows[sg.kind];
            const int at = ALONE ? tile0 + tl : piece * (rows >> 1) + tl;
            float4* prow = p.part_o[sg.kind] + (size_t)sg.slot * (D / 4) * rows + at;
            float2* pml = p.part_ml[sg.kind] + (size_t)sg.slot * rows + at;
            live = si.next(sg);
            if (live) q_ask();
            if (!ok || !(ok = mbar_wait_warp(bar(X_OFULL + x), o_phase, abort_flag))) break;
            float2 ml = make_float2(l_run > 0.f ? m_ref : -INFINITY, l_run);
            // O is free for the next segment's products as soon as it has been read, ahead of the last stores.  (The arrival releases: the
            // loads from tensor memory are done, tcgen05.wait::ld, and ordered ahead of it.  That it also orders the partials stored
            // before it cost nothing on the listed shapes.)
            if (ALONE && alt) {
                // Both tiles have a part of every row; each adds up half of the columns.  (The statistics of the last alternate segment
                // have been read by everybody: O is complete only after both tiles have let go of the last one's.)
                if (!(ok = mbar_wait_warp(bar(X_OFULL + (x ^ 1)), o_phase, abort_flag))) break;
                float2* stat = reinterpret_cast<float2*>(sm + SMEM_STAT);
                stat[x * 128 + tl] = ml;
                mbar_arrive(bar(X_STAT));
                if (!(ok = mbar_wait_warp(bar(X_STAT), stat_phase, abort_flag))) break;
                stat_phase ^= 1;
                const float2 other = stat[(x ^ 1) * 128 + tl];
                const float m = fmaxf(ml.x, other.x), m_use = m == -INFINITY ? 0.f : m;
                const float w = exp2f(ml.x - m_use), u = exp2f(other.x - m_use);          // 0 for a tile that saw nothing
                ml = make_float2(m, ml.y * w + other.y * u);
                tc_fence_after();
                if (warp_rows) {
                    const uint32_t from = x * 64, peer = lane_addr + COL_O + (x ^ 1) * 128;
                    prow += (size_t)(x * 16) * rows;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t o[32], q[32];
                        tmem_ld32(o_addr + from + c * 32, o);
                        tmem_ld32(peer + from + c * 32, q);
                        tmem_wait_ld();
                        if (c == 1) { tc_fence_before(); mbar_arrive(bar(X_OFREE + x)); }
                        if (row_ok) {
#pragma unroll
                            for (int c4 = 0; c4 < 8; ++c4, prow += rows) {
                                float v[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e)      // (undefined where no product ran)
                                    v[e] = (w > 0.f ? w * __uint_as_float(o[4 * c4 + e]) : 0.f) + (u > 0.f ? u * __uint_as_float(q[4 * c4 + e]) : 0.f);
                                *prow = make_float4(v[0], v[1], v[2], v[3]);
                            }
                        }
                    }
                } else {
                    mbar_arrive(bar(X_OFREE + x));
                }
            } else {
                tc_fence_after();
                if (warp_rows) {
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) {
                        uint32_t o[32];
                        tmem_ld32(o_addr + c * 32, o);
                        tmem_wait_ld();
                        if (c == D / 32 - 1) { tc_fence_before(); mbar_arrive(bar(X_OFREE + x)); }
                        if (row_ok && has_o) {                // (without a product the piece has l = 0 and its o is not looked at)
#pragma unroll
                            for (int c4 = 0; c4 < 8; ++c4, prow += rows)
                                *prow = make_float4(__uint_as_float(o[4 * c4]), __uint_as_float(o[4 * c4 + 1]), __uint_as_float(o[4 * c4 + 2]), __uint_as_float(o[4 * c4 + 3]));
                        }
                    }
                } else {
                    mbar_arrive(bar(X_OFREE + x));
                }
            }
            if (row_ok && (!(ALONE && alt) || x == 0)) *pml = ml;
            o_phase ^= 1;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(*tmem_slot), "r"(TMEM_COLS) : "memory");
    }
    if (tid == 0 && *abort_flag) atomicCAS(p.status, 0, (int)VISPEC_E_TIMEOUT);
}

// The pieces of a row added up: a thread has C4 groups of four columns of one row; the lanes of a warp have consecutive rows of a
// (sequence, kv head), which lie side by side in the partials of both kinds.  Four pieces at a time, their loads ahead of the sums.
template <int C4>
__global__ void __launch_bounds__(128)
prefix_merge_kernel(const __grid_constant__ PrefixParams p) {
    const int lane = threadIdx.x & 31;
    pdl_launch_dependents();
    const int RG = p.N * p.G, CG = D / 4 / C4;
    const long long idx = (long long)blockIdx.x * 128 + threadIdx.x, all = (long long)p.B * p.Hkv * RG * CG;
    const bool live = idx < all;
    const long long li = live ? idx : all - 1;
    const int r = (int)(li % RG), cg = (int)(li / RG % CG), kvh = (int)(li / RG / CG % p.Hkv), b = (int)(li / RG / CG / p.Hkv);
    // the line, from kv_len, which the attention kernel does not write: every lane takes part in the sums, then takes its sequence's
    int kv[kMaxLineB / 32], at[kMaxLineB / 32], own[kMaxLineB / 32];
    if (!p.early) pdl_wait();
#pragma unroll
    for (int i = 0; i < kMaxLineB / 32; ++i) { kv[i] = i * 32 + lane < p.B ? p.kv_len[i * 32 + lane] : 0; at[i] = 0; own[i] = -1; }
    const int T = line_build(p, lane, kv, [&](int i, int, int place, int S) { at[i] = place; own[i] = S; });
    int base_b = 0, S = -1;
#pragma unroll
    for (int i = 0; i < kMaxLineB / 32; ++i) {
        const int x = __shfl_sync(0xffffffffu, at[i], b & 31), y = __shfl_sync(0xffffffffu, own[i], b & 31);
        if (b >> 5 == i) { base_b = x; S = y; }
    }
    const int R = range_of(p, T);
    const int node = r / p.G, head = kvh * p.G + r % p.G;
    int n[2], first[2];                                   // pieces of a kind, row of the first one in its region
    bool two[2] = {false, false};                         // two pieces to a slot
#pragma unroll
    for (int kind = 0; kind < 2; ++kind) {
        const int keys = kind ? S + p.N : p.P, steps = S < 0 ? 0 : steps_of(keys), row = kind ? r : b * RG + r;
        const int m = row / kRows, nb = p.blocks[kind];
        n[kind] = first[kind] = 0;
        if (steps == 0) continue;
        const bool alt = m == nb - 1 && p.last_alt[kind];
        const int u0 = (kind ? base_b : 0) + kvh * head_places(p, kind, steps) + m * unit_places(p, kind, steps, false) + start_places(alt);
        const int c0 = u0 / R, unit = kind ? (b * p.Hkv + kvh) * nb + m : kvh * nb + m;
        const int lr = row - m * kRows;
        two[kind] = alt && steps > 1;                     // (an alternate unit of one step: the second tile has nothing)
        n[kind] = ((u0 + (steps - 1) * step_places(alt)) / R - c0 + 1) << (two[kind] ? 1 : 0);
        first[kind] = (unit + c0) * p.slot_rows[kind] + (lr < 128 ? lr : (p.slot_rows[kind] >> 1) + lr - 128);
    }
    if (p.early) pdl_wait();
    if (!live) return;
    float m_all = -INFINITY, l_all = 0.f;
    float4 acc[C4];
#pragma unroll
    for (int k = 0; k < C4; ++k) acc[k] = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr int U = C4 == 1 ? 8 : 4;
    const int entries = n[0] + n[1];
    for (int e0 = 0; e0 < entries; e0 += U) {
        float2 ml[U];
        float4 v[U][C4];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = e0 + u;
            ml[u] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int k = 0; k < C4; ++k) v[u][k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (e < entries) {
                const bool own = e >= n[0];
                const int rows = own ? p.slot_rows[1] : p.slot_rows[0], ek = own ? e - n[0] : e;
                const int pos = (own ? first[1] : first[0]) + ((own ? two[1] : two[0]) ? ek * (rows >> 1) : ek * rows);
                const int slot = pos / rows, in = pos - slot * rows;
                ml[u] = __ldcg((own ? p.part_ml[1] : p.part_ml[0]) + pos);
                const float4* src = (own ? p.part_o[1] : p.part_o[0]) + ((size_t)slot * (D / 4) + cg * C4) * rows + in;
#pragma unroll
                for (int k = 0; k < C4; ++k) v[u][k] = __ldcg(src + (size_t)k * rows);
            }
        }
        float m_new = m_all;
#pragma unroll
        for (int u = 0; u < U; ++u) m_new = fmaxf(m_new, ml[u].x);
        const float m_fin = (m_new == -INFINITY) ? 0.f : m_new;
        const float a = exp2f(m_all - m_fin);                 // 0 while nothing has been accumulated
        l_all *= a;
#pragma unroll
        for (int k = 0; k < C4; ++k) { acc[k].x *= a; acc[k].y *= a; acc[k].z *= a; acc[k].w *= a; }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float w = exp2f(ml[u].x - m_fin);           // 0 for a piece that saw nothing (or is absent)
            l_all += ml[u].y * w;
            if (ml[u].x == -INFINITY) continue;               // (its o may never have been written)
#pragma unroll
            for (int k = 0; k < C4; ++k) { acc[k].x += w * v[u][k].x; acc[k].y += w * v[u][k].y; acc[k].z += w * v[u][k].z; acc[k].w += w * v[u][k].w; }
        }
        m_all = m_new;
    }
    const float inv = inv_sum(l_all);
    __nv_bfloat16* orow = p.out + (((size_t)b * p.N + node) * p.Hq + head) * D + cg * C4 * 4;
    if constexpr (C4 == 1) {
        *reinterpret_cast<uint2*>(orow) = make_uint2(pack_bf16(acc[0].x * inv, acc[0].y * inv), pack_bf16(acc[0].z * inv, acc[0].w * inv));
    } else {
#pragma unroll
        for (int k = 0; k < C4; k += 2)
            *reinterpret_cast<uint4*>(orow + k * 4) =
                make_uint4(pack_bf16(acc[k].x * inv, acc[k].y * inv), pack_bf16(acc[k].z * inv, acc[k].w * inv),
                           pack_bf16(acc[k + 1].x * inv, acc[k + 1].y * inv), pack_bf16(acc[k + 1].z * inv, acc[k + 1].w * inv));
    }
    if (p.lse && cg == 0)
        p.lse[((size_t)b * p.Hq + head) * p.N + node] = l_all > 0.f ? (m_all + log2f(l_all)) * 0.6931471805599453f : -INFINITY;
    if (S < 0 && cg == 0 && r == 0 && kvh == 0) atomicCAS(p.status, 0, (int)VISPEC_E_RANGE);
}

// ------------------------------------------------------------------------------------------------
// Few rows per unit (N * G <= 8: single tokens, small trees): the sequences' own keys, and the join with the prefix.
//
// What bounds it: the read of the own keys.  A tile of 128 rows would be nearly empty and its segments would cost more to start than
// to stream (32 sequences x 40 heads with one row each: 8 segments per SM of 8 to 10 thousand cycles), so here a warp takes 16 keys at
// a time on its own, by asynchronous 16-byte copies into shared memory of its own, a group ahead, and has no barrier to set up:
//   S = Q K^T   (mma.sync m16n8k16) lane (key k = lane / 4, part q = lane % 4) reads 16 bytes of key k at elements 32 j + 8 q: the pairs
//               are the B operand of two products whose 16 contracted elements are 32 j + 8 q' + 4 s + {0, 1} and + {2, 3}; Q alike.
//   O += P V    P is S's accumulator layout read as an A operand.  The lane reads 16 bytes of keys 2q, 2q + 1, 2q + 8, 2q + 9 at
//               elements 64 h + 8 (lane / 4); column c of product (h, t) is element 64 h + 8 c + t, so a lane's accumulators are 16
//               consecutive elements of each half of its rows.
// (Loaded straight into registers instead, 12 warps of 168 registers per SM reached 3.7 TB/s: a warp then either loads or computes.)
// A unit is a warp's, or that of 2 or 4 warps of a block, or where units are few of a cluster of 2, 4 or 8 blocks; they take the groups
// of 16 keys and the prefix's pieces in turn, their (m, l, o) meet in shared memory, behind a barrier of the block or two of the
// cluster, and the row is finished here.  (Three blocks per SM leave 168 registers a thread; the assembler spills 36 bytes, in the
// join of the prefix's pieces.)
// ------------------------------------------------------------------------------------------------
constexpr int kFewWarps = 4, kFewRows = 8, kFewStages = 2;
constexpr int kFewStage = 2 * 16 * D * 2;          // bytes of 16 keys and their values
constexpr int kFewSmem = kFewWarps * kFewStages * kFewStage;

__device__ __forceinline__ void mma_16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// (Units of 9 to 16 rows the same way, two accumulators a lane and the registers of two blocks per SM, were no faster than on the line:
// 16 x 2 nodes of 16/2 heads on 3000 + 1000 keys 25.9 us against 18.1, 24 x 16 of 32/32 on 2000 + 1500 131 against 109.)
__global__ void __launch_bounds__(32 * kFewWarps, 3)
few_rows_kernel(const __grid_constant__ PrefixParams p, const __grid_constant__ PagedArgs pa, const uint4* __restrict__ k_pool,
                const uint4* __restrict__ v_pool, const int wpu /* warps of a block that share a unit */) {
    constexpr int ROWS = 8;
    extern __shared__ __align__(1024) unsigned char sm[];
    __shared__ float2 park_ml[kFewWarps][ROWS];
    static_assert(ROWS * (D / 4 + 1) * 16 <= kFewStages * kFewStage, "a warp's part does not fit its stages");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q4 = lane & 3, c8 = lane >> 2;
    const int ck = (int)cluster_size(), cr = (int)cluster_ctarank();
    const int sub = warp % wpu, first_warp = warp - sub, units = p.B * p.Hkv;
    const int unit_ = ck > 1 ? blockIdx.x / ck : (blockIdx.x * kFewWarps + warp) / wpu;
    const bool live = unit_ < units;               // (the last block may have warps without a unit)
    const int unit = live ? unit_ : units - 1, b = unit / p.Hkv, kvh = unit - b * p.Hkv;
    const int wi = ck > 1 ? cr * kFewWarps + warp : sub, nw = ck > 1 ? ck * kFewWarps : wpu;
    const int RG = p.N * p.G;
    if (!p.early) pdl_wait();
    pdl_launch_dependents();
    const int S = own_len(p, p.kv_len[b]), total = S + p.N;
    const bool good = S >= 0;
    // The lane's row is c8.  (q, tree_mask and the tree's own keys: the kernel before has waited for what
    // writes them before it let this one in; where there is none, this one waits.)
    if (p.early && p.P == 0) pdl_wait();
    const bool there = c8 < RG;
    const int node = there ? c8 / p.G : 0;
    uint32_t qa[D / 16][2];                        // [2 j + s]: A registers of the row, first and second half of the 16 elements
    {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (((size_t)b * p.N + node) * p.Hq + kvh * p.G + (there ? c8 % p.G : 0)) * D) + q4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 v = there ? __ldcg(src + 4 * j) : make_uint4(0, 0, 0, 0);
            qa[2 * j][0] = v.x; qa[2 * j][1] = v.y; qa[2 * j + 1][0] = v.z; qa[2 * j + 1][1] = v.w;
        }
    }
    const uint64_t mk = there ? __ldcg(p.mask + (size_t)b * p.N + node) : 0ull;              // (N <= 8: one word)
    float o[16][2], m_ref = -INFINITY, l_run = 0.f;                                          // o[t + 8 h][i]: element 64 h + 8 (2 q4 + i) + t
#pragma unroll
    for (int t = 0; t < 16; ++t) o[t][0] = o[t][1] = 0.f;

    // ---- own keys: groups of 16, number i of this warp is wi + i * nw ----
    const int groups = good && live ? (total + 15) / 16 : 0, mine_n = groups > wi ? (groups - wi + nw - 1) / nw : 0;
    const int32_t* trow = pa.block_table + (size_t)b * pa.table_stride + p.P / pa.page_rows;
    const size_t stride = (size_t)(pa.token_major ? pa.Hkv : 1) * (D / 8);                  // 16-byte vectors between keys
    const size_t head_at = (size_t)kvh * (pa.token_major ? 1 : pa.page_rows) * (D / 8);
    const size_t block = (size_t)pa.page_rows * pa.Hkv * (D / 8);
    unsigned char* const mine = sm + warp * kFewStages * kFewStage;
    const uint32_t mine_at = smem_u32(mine);
    // the table's entries of the warp's groups 32 i .. 32 i + 31, asked for ahead of kv_len
    auto entries_at = [&](int i) {
        const int at = (wi + (i + lane) * nw) * 16 / pa.page_rows;
        return at < pa.table_stride - p.P / pa.page_rows ? trow[at] : -1;
    };
    int entries = entries_at(0);
    // Group i on its way into stage i % kFewStages: half a warp per key, 16-byte chunks exchanged so that the reads below
    // meet every bank once.  Keys past the last one (their rows may hold anything) and entries outside the pool become zeros.
    auto fetch = [&](int i) {
        if (i < mine_n) {
            if (i > 0 && (i & 31) == 0) entries = entries_at(i);
            const int e = __shfl_sync(0xffffffffu, entries, i & 31), key0 = (wi + i * nw) * 16;
            const bool in_pool = e >= 0 && e < pa.num_blocks;
            if (!in_pool && lane == 0 && p.status) atomicCAS(p.status, 0, (int)VISPEC_E_RANGE);
            const int c = lane & 15, r0 = lane >> 4;
            const size_t at = (in_pool ? (size_t)e : 0) * block + head_at + (size_t)(key0 % pa.page_rows + r0) * stride + c;
            const uint32_t dst = mine_at + (uint32_t)(i % kFewStages) * kFewStage;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int r = 2 * k + r0, n = in_pool && key0 + r < total ? 16 : 0;
                const size_t from = n ? at + 2 * k * stride : 0;
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + r * 256 + ((c ^ (4 * (r & 1))) << 4)), "l"(k_pool + from), "r"(n) : "memory");
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + kFewStage / 2 + r * 256 + ((c ^ (2 * ((r >> 1) & 3))) << 4)), "l"(v_pool + from), "r"(n) : "memory");
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kFewStages - 1; ++i) fetch(i);
    for (int i = 0; i < mine_n; ++i) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 2) : "memory");
        __syncwarp();                              // everybody's copies of this group are here, and nobody reads the last one any more
        fetch(i + kFewStages - 1);
        const int key0 = (wi + i * nw) * 16;
        const unsigned char* ks = mine + i % kFewStages * kFewStage;
        const unsigned char* vs = ks + kFewStage / 2;
        float sc[2][4];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 kk = *reinterpret_cast<const uint4*>(ks + (8 * n + c8) * 256 + (((4 * j + q4) ^ (4 * (c8 & 1))) << 4));
                const uint32_t a0[4] = {qa[2 * j][0], 0u, qa[2 * j][1], 0u}, a1[4] = {qa[2 * j + 1][0], 0u, qa[2 * j + 1][1], 0u};
                mma_16816(sc[n], a0, kk.x, kk.y);
                mma_16816(sc[n], a1, kk.z, kk.w);
            }
        }
        float x[4] = {sc[0][0], sc[0][1], sc[1][0], sc[1][1]};                               // keys 2q, 2q+1, 2q+8, 2q+9
        if (key0 + 16 > S) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int t = key0 + 2 * q4 + (k & 1) + 8 * (k >> 1) - S;                   // tree node of this key, if it is one
                if (t >= 0 && !(t < p.N && (mk >> t) & 1ull)) x[k] = -INFINITY;
            }
        }
        float top = max_nan(max3_nan(x[0], x[1], x[2]), x[3]);
        top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2)) * p.scale_log2;
        if (top > m_ref + kRescaleGap) {                                                     // also on the first finite group
            const float a = exp2f(m_ref - top);
            m_ref = top;
            l_run *= a;
#pragma unroll
            for (int t = 0; t < 16; ++t) { o[t][0] *= a; o[t][1] *= a; }
        }
        if (!(top < INFINITY)) l_run = top - top;                                            // a NaN or an infinite score (see inv_sum)
        const float m_use = m_ref == -INFINITY ? 0.f : m_ref;
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = exp2f(fmaf(x[k], p.scale_log2, -m_use));
        l_run += (x[0] + x[1]) + (x[2] + x[3]);                                              // this lane's keys; summed over the lanes below
        const uint32_t pr[4] = {pack_bf16(x[0], x[1]), 0u, pack_bf16(x[2], x[3]), 0u};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t v[4][4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const uint4 u = *reinterpret_cast<const uint4*>(vs + (2 * q4 + (x & 1) + 8 * (x >> 1)) * 256 + (((8 * h + c8) ^ (2 * q4)) << 4));
                v[x][0] = u.x; v[x][1] = u.y; v[x][2] = u.z; v[x][3] = u.w;
            }
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                const uint32_t sel = t & 1 ? 0x7632u : 0x5410u;
                float c[4] = {o[8 * h + t][0], o[8 * h + t][1], 0.f, 0.f};
                mma_16816(c, pr, __byte_perm(v[0][t >> 1], v[1][t >> 1], sel), __byte_perm(v[2][t >> 1], v[3][t >> 1], sel));
                o[8 * h + t][0] = c[0]; o[8 * h + t][1] = c[1];
            }
        }
    }
    __syncwarp();                                  // (the stages take the warp's part below)
    // (a NaN or infinite score was seen by all lanes of the row, so every lane's l is NaN then)
    l_run += __shfl_xor_sync(0xffffffffu, l_run, 1);
    l_run += __shfl_xor_sync(0xffffffffu, l_run, 2);
    if (!(l_run > 0.f)) m_ref = -INFINITY;

    // ---- the prefix's pieces of the row, from the kernel before ----
    if (p.early && p.P > 0) pdl_wait();
    if (good && live && p.P > 0) {
        const int steps = steps_of(p.P), Rg = range_of(p, p.Hkv * head_places(p, 0, steps)), rows = p.slot_rows[0];
        const int row = b * RG + min(c8, RG - 1), m = row / kRows, lr = row - m * kRows, nb = p.blocks[0];
        const bool alt = m == nb - 1 && p.last_alt[0];
        const int u0 = kvh * head_places(p, 0, steps) + m * unit_places(p, 0, steps, false) + start_places(alt);
        const int first = u0 / Rg, last = (u0 + (steps - 1) * step_places(alt)) / Rg;
        const int pieces = last - first + 1;
        for (int e0 = wi; e0 < pieces; e0 += 2 * nw) {                                       // two at a time, their loads ahead of the sums
            float2 ml[2];
            float4 v[2][8];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int e = e0 + k * nw < pieces ? e0 + k * nw : e0;
                const int slot = kvh * nb + m + first + e;
                ml[k] = __ldcg(p.part_ml[0] + (size_t)slot * rows + lr);
                const float4* src = p.part_o[0] + ((size_t)slot * (D / 4) + 4 * q4) * rows + lr;
#pragma unroll
                for (int x = 0; x < 8; ++x) v[k][x] = __ldcg(src + (size_t)((x & 3) + 16 * (x >> 2)) * rows);
            }
            if (e0 + nw >= pieces) ml[1] = make_float2(-INFINITY, 0.f);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const float m_new = fmaxf(m_ref, ml[k].x), m_use = m_new == -INFINITY ? 0.f : m_new;
                const float a = exp2f(m_ref - m_use), w = exp2f(ml[k].x - m_use);
                l_run = l_run * a + ml[k].y * w;
                m_ref = m_new;
                if (ml[k].x == -INFINITY) continue;                                          // (its o may never have been written)
#pragma unroll
                for (int x = 0; x < 8; ++x) {                                                // elements 64 h + 16 q4 + 4 (x & 3) + 0..3
                    const int h = x >> 2, i = (x & 3) >> 1, t = 8 * h + 4 * (x & 1);
                    o[t][i] = o[t][i] * a + v[k][x].x * w;
                    o[t + 1][i] = o[t + 1][i] * a + v[k][x].y * w;
                    o[t + 2][i] = o[t + 2][i] * a + v[k][x].z * w;
                    o[t + 3][i] = o[t + 3][i] * a + v[k][x].w * w;
                }
            }
        }
    }

    // ---- the warps' parts meet ----
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        const int h = x >> 2, i = (x & 3) >> 1, t = 8 * h + 4 * (x & 1);
        reinterpret_cast<float4*>(mine)[c8 * (D / 4 + 1) + 16 * h + 4 * q4 + (x & 3)] = make_float4(o[t][i], o[t + 1][i], o[t + 2][i], o[t + 3][i]);
    }
    if (q4 == 0) park_ml[warp][c8] = make_float2(m_ref, l_run);
    if (ck > 1) cluster_sync_all(); else if (wpu > 1) __syncthreads(); else __syncwarp();
    const uint32_t o_at = smem_u32(sm), ml_at = smem_u32(&park_ml[0][0]);
    // thread <-> (row, 4 columns); the ranks of a cluster take rows in turn
    for (int item = wi * 32 + lane; live && item < RG * (D / 4); item += nw * 32) {
        const int row = item / (D / 4), c4 = item % (D / 4);
        float m_all = -INFINITY, l_all = 0.f;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int k = 0; k < ck; ++k) {
            float2 ml[kFewWarps];
            float4 v[kFewWarps];
            const uint32_t po = ck > 1 ? dsmem_addr(o_at, k) : o_at, pm = ck > 1 ? dsmem_addr(ml_at, k) : ml_at;
#pragma unroll
            for (int x = 0; x < kFewWarps; ++x) {
                const int w = first_warp + x;
                ml[x] = make_float2(-INFINITY, 0.f);
                v[x] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (x >= wpu) continue;
                const uint32_t om = (uint32_t)((w * ROWS + row) * 8), oo = (uint32_t)(w * kFewStages * kFewStage + (row * (D / 4 + 1) + c4) * 16);
                ml[x] = ck > 1 ? dsmem_ld2(pm + om) : smem_ld2(pm + om);
                v[x] = ck > 1 ? dsmem_ld4(po + oo) : smem_ld4(po + oo);
            }
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) {
                const float m_new = fmaxf(m_all, ml[w].x), m_use = m_new == -INFINITY ? 0.f : m_new;
                const float a = exp2f(m_all - m_use), u = exp2f(ml[w].x - m_use);
                l_all = l_all * a + ml[w].y * u;
                acc.x = acc.x * a + v[w].x * u; acc.y = acc.y * a + v[w].y * u; acc.z = acc.z * a + v[w].z * u; acc.w = acc.w * a + v[w].w * u;
                m_all = m_new;
            }
        }
        const int node = row / p.G, head = kvh * p.G + row % p.G;
        const float inv = inv_sum(l_all);
        *reinterpret_cast<uint2*>(p.out + (((size_t)b * p.N + node) * p.Hq + head) * D + c4 * 4) =
            make_uint2(pack_bf16(acc.x * inv, acc.y * inv), pack_bf16(acc.z * inv, acc.w * inv));
        if (p.lse && c4 == 0)
            p.lse[((size_t)b * p.Hq + head) * p.N + node] = l_all > 0.f ? (m_all + log2f(l_all)) * 0.6931471805599453f : -INFINITY;
    }
    if (!good && kvh == 0 && wi == 0 && lane == 0) atomicCAS(p.status, 0, (int)VISPEC_E_RANGE);
    if (ck > 1) cluster_sync_all();                // nobody leaves while a peer may still read its shared memory
}

// What of the scratch a call of B sequences of N nodes uses.
struct PrefixLayout {
    int rows[2], blocks[2], slot_rows[2];
    long long slots[2];
    size_t bytes[2];
};
PrefixLayout prefix_layout(int B, int N, int Hq, int Hkv, int sm_count, bool alone) {
    PrefixLayout l;
    const int G = Hq / Hkv;
    for (int kind = 0; kind < 2; ++kind) {
        l.rows[kind] = (kind ? N : B * N) * G;
        l.blocks[kind] = (l.rows[kind] + kRows - 1) / kRows;
        const int rows8 = (l.rows[kind] + 7) / 8 * 8;
        l.slot_rows[kind] = l.rows[kind] > 128 ? (alone && rows8 < kRows ? rows8 : kRows) : alone ? rows8 : 2 * rows8;
        l.slots[kind] = kind && alone ? 0 : (long long)(kind ? B : 1) * Hkv * l.blocks[kind] + sm_count;     // (few_rows_kernel parks nothing)
        l.bytes[kind] = (size_t)l.slots[kind] * l.slot_rows[kind] * (D * 4 + 8);
    }
    return l;
}

}  // namespace

// The larger of what the two ways take where either may be chosen, so that it is never less for more sequences.
size_t prefix_scratch_bytes(int B, int N, int Hq, int Hkv, int sm_count) {
    const bool few = N * (Hq / Hkv) <= kFewRows;
    const PrefixLayout line = prefix_layout(few ? std::min(B, kMaxLineB) : B, N, Hq, Hkv, sm_count, false);
    const PrefixLayout alone = prefix_layout(B, N, Hq, Hkv, sm_count, true);
    return std::max(line.bytes[0] + line.bytes[1], few ? alone.bytes[0] : 0);
}

// Keys of its own that a sequence may have, as far as the host can tell: what the hint says (a committed length, the prefix and all; one
// below the prefix is none of this call's sequences'), or else all that the table has room for.
static int own_keys(const AttnArgs& a, int prefix) {
    const int cap = a.S_max - prefix;
    if (a.kv_len_hint <= 0 || a.kv_len_hint < prefix) return cap;
    return (int)std::min((long long)cap, (long long)a.kv_len_hint - prefix + a.N);
}
// Do the sequences' own keys go through few_rows_kernel?  Short ones do, and long ones where the prefix outweighs them all; long
// own keys stream better on the line.  us, few_rows_kernel / line, sequences x nodes of heads on prefix + own keys:
//   won   32 x 1 of 40/40 on 2880 + 200     47.4 / 66.7    2 x 1 of 40/40 on 2880 + 200   22.9 / 27.4    24 x 1 of 32/8 on 3000 + 100  16.5 / 18.9
//         8 x 1 of 28/4 on 3344 + 200       14.6 / 15.6    32 x 1 of 28/4 on 3344 + 200   19.0 / 19.4    8 x 1 of 32/32 on 2000 + 500  29.7 / 30.9
//         8 x 1 of 16/2 on 32768 + 1000     28.1 / 54.2
//   lost  2 x 1 of 28/4 on 1000 + 100       13.2 / 10.7    2 x 8 of 32/32 on 3000 + 300   25.0 / 19.9    20 x 1 of 16/2 on 2000 + 300  14.1 / 13.3
//         4 x 2 of 32/8 on 2000 + 300       13.7 / 13.2    4 x 1 of 32/8 on 1000 + 800    13.9 / 13.1    8 x 4 of 32/32 on 3000 + 300  28.1 / 26.8
//         16 x 1 of 32/32 on 2000 + 500     44.0 / 43.5    16 x 8 of 32/32 on 3000 + 300  44.1 / 43.2
//   longer own keys (an earlier form of this kernel): 40 x 1 of 28/4 on 2000 + 2000 46 / 34, 48 x 1 of 32/8 on 1000 + 2000 73 / 69
// The rule knows the lengths only, so calls of few units are up to a quarter slower than they could be.
static bool few_rows(const AttnArgs& a, int prefix) {
    if (a.N * (a.Hq / a.Hkv) > kFewRows) return false;
    const int own = own_keys(a, prefix);
    return a.B > kMaxLineB || own <= 1024 || (long long)a.B * own <= prefix;
}

cudaError_t init_attn_prefix() {
    const void* merges[2] = {(const void*)prefix_merge_kernel<1>, (const void*)prefix_merge_kernel<4>};
    for (const void* m : merges) {                    // (see init_merge)
        const cudaError_t e = cudaFuncSetAttribute(m, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
        if (e != cudaSuccess) return e;
    }
    const cudaError_t f = cudaFuncSetAttribute((const void*)few_rows_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kFewSmem);
    if (f != cudaSuccess) return f;
    const cudaError_t e = cudaFuncSetAttribute((const void*)attn_prefix_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_ALLOC);
    return e != cudaSuccess ? e : cudaFuncSetAttribute((const void*)attn_prefix_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_ALLOC);
}

// Sizes that these kernels take: every place of the line and every row of the partials has a 32-bit number.
bool attn_prefix_supports(const AttnArgs& a, int prefix) {
    const bool few = few_rows(a, prefix);
    if ((!few && a.B > kMaxLineB) || !(a.scale > 0.f) || a.D != D || !a.page_rows) return false;
    const PrefixLayout l = prefix_layout(a.B, a.N, a.Hq, a.Hkv, a.sm_count, few);
    long long T = 0;
    for (int kind = 0; kind < (few ? 1 : 2); ++kind) {
        const long long steps = ((kind ? (long long)a.S_max - prefix : prefix) + STEP - 1) / STEP;
        T += (kind ? (long long)a.B : 1) * a.Hkv * l.blocks[kind] * (kWideStart + steps * kWideStep);
        if (l.slots[kind] * l.slot_rows[kind] >= (1ll << 31)) return false;
    }
    return T < (1ll << 31) - (1 << 20);
}

cudaError_t launch_attn_prefix(const AttnArgs& a, int prefix, void* scratch, cudaStream_t st, int* n_launches) {
    const bool few = few_rows(a, prefix);
    const PrefixLayout l = prefix_layout(a.B, a.N, a.Hq, a.Hkv, a.sm_count, few);
    PrefixParams p = {};
    p.q = (const __nv_bfloat16*)a.q; p.kv_len = a.kv_len; p.mask = a.mask;
    p.out = (__nv_bfloat16*)a.out; p.lse = a.lse;
    unsigned char* ws = (unsigned char*)scratch;
    for (int kind = 0; kind < 2; ++kind) {
        p.part_o[kind] = (float4*)ws;
        ws += (size_t)l.slots[kind] * l.slot_rows[kind] * D * 4;
        p.slot_rows[kind] = l.slot_rows[kind]; p.blocks[kind] = l.blocks[kind];
        p.last_alt[kind] = l.rows[kind] - (l.blocks[kind] - 1) * kRows <= 128;
    }
    for (int kind = 0; kind < 2; ++kind) { p.part_ml[kind] = (float2*)ws; ws += (size_t)l.slots[kind] * l.slot_rows[kind] * 8; }
    p.B = a.B; p.N = a.N; p.Hq = a.Hq; p.Hkv = a.Hkv; p.G = a.Hq / a.Hkv;
    p.P = prefix; p.cap = a.S_max - prefix;
    p.early = a.early_prefetch ? 1 : 0; p.grid = a.sm_count; p.groups = a.B;
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.status = a.status;
    const PagedArgs pa = {a.block_table, a.table_stride, a.page_rows, a.num_blocks, a.Hkv, a.N, a.token_major, a.status, nullptr};
    if (few) {
        p.groups = 0;
        // More SMs than ranges worth having: a unit is cut into equal parts of whole ranges, so that no CTA starts on a second unit
        // while others have none.
        const int steps = steps_of(prefix), n = a.Hkv * l.blocks[0], len = unit_places(p, 0, steps, l.blocks[0] == 1);
        if (steps > 0 && n <= a.sm_count && a.Hkv * head_places(p, 0, steps) < a.sm_count * kMinRange) {
            const int parts = std::max(1, std::min(a.sm_count / n, len / kMinRange));
            p.range = (len + parts - 1) / parts;
            p.pad = parts * p.range;
        }
    }
    cudaError_t err = cudaSuccess;
    if (!few || prefix > 0) {
        err = few ? launch_pdl(attn_prefix_kernel<true>, dim3(p.grid), dim3(kThreads), SMEM_ALLOC, st, 0, *a.k_map, *a.v_map, p, pa)
                  : launch_pdl(attn_prefix_kernel<false>, dim3(p.grid), dim3(kThreads), SMEM_ALLOC, st, 0, *a.k_map, *a.v_map, p, pa);
        if (err != cudaSuccess) return err;
        ++*n_launches;
    }
    if (few) {
        // Warps to a unit: as many as the SMs hold at once, as long as each has a group of keys or a piece of the prefix, or in a cluster
        // four of them (4 x 2 of 32/8 heads on 2000 + 300 keys: 13.4 us with 4 warps, 17.0 with 16; 4 x 1 of 28/4 on 16 + 4000: 55.7, 18.5 with 32).
        const int units = a.B * a.Hkv, steps = steps_of(prefix), T = a.Hkv * head_places(p, 0, steps), room = 12 * a.sm_count;
        const int pieces = steps == 0 ? 0 : unit_places(p, 0, steps, true) / range_of(p, T) + 1, most = std::max((own_keys(a, prefix) + 15) / 16, pieces);
        int nw = 1;
        while (nw < 8 * kFewWarps && (nw < kFewWarps ? 2 : 8) * nw <= most && units * 2 * nw <= room) nw *= 2;
        const int ck = nw > kFewWarps ? nw / kFewWarps : 1, wpu = nw > kFewWarps ? kFewWarps : nw;
        const int blocks = ck > 1 ? units * ck : (units * wpu + kFewWarps - 1) / kFewWarps;
        err = launch_pdl(few_rows_kernel, dim3(blocks), dim3(32 * kFewWarps), kFewSmem, st, ck, p, pa, (const uint4*)a.k, (const uint4*)a.v, wpu);
        if (err == cudaSuccess) ++*n_launches;
        return err;
    }
    // One group of four columns per thread while that leaves the SMs with few threads, whole 32-byte sectors of the output beyond
    // (8 x 60 nodes of 32/32 heads: 60.9 us, one group each 68.8).
    const long long rows = (long long)a.B * a.N * a.Hq;
    const bool fine = rows * (D / 4) <= 1024ll * a.sm_count;
    const unsigned blocks = (unsigned)((rows * (fine ? D / 4 : D / 16) + 127) / 128);
    err = fine ? launch_pdl(prefix_merge_kernel<1>, dim3(blocks), dim3(128), 0, st, 0, p)
               : launch_pdl(prefix_merge_kernel<4>, dim3(blocks), dim3(128), 0, st, 0, p);
    if (err == cudaSuccess) ++*n_launches;
    return err;
}

}  // namespace vispec
