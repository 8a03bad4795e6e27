// Decode attention over rows that a group of sequences has in common (Eq. 1 of the paper, block tables): read once for all of
// them.  For the query rows i of a group's members (member by member, the G heads of a KV head side by side) and a run of the
// common rows,
//   l_i = sum_n 2^(s_in - m_i),  o_i = sum_n 2^(s_in - m_i) V_n,   s_in = scale log2(e) q_i . K_n,  m_i >= max_n s_in,
// which dense_kernel joins with the sequences' own rows.
//
//   - A workgroup of four waves has a tile of 64 WQ query rows and a run of rows.  A wave holds 64 query rows (operands and sums:
//     192 registers) and goes over 32 rows at a time on v_mfma_f32_32x32x16_bf16: S^T = K Q^T, O^T += V^T P^T.  In S^T a lane has 16
//     rows of ONE query row, which are what the second product wants from it as P: nothing crosses lanes.
//   - WQ waves share what they read (rows come into LDS by direct loads, 64 of K and of V a stage), 4 / WQ go over different rows.
//   - The maximum is followed loosely: scaling a wave's sums takes 1500 cycles, as much as two thirds of the products of 32 rows, so the
//     reference m_i is set PREFIX_LOOSE (binary) orders above the highest score when one passes it.  Weights are at most 1 all the same,
//     and as floating-point numbers keep their precision; what is lost are weights 2^-70 of the largest, and values below 2^-70.
//     (32 sequences behind 32768 rows, 256 heavy ones behind 16384, us with 32, 40 and 56 orders: 77.9 / 74.0 / 70.8, 282 / 277 / 274)
//   - A weight is two bf16 terms, the upper half of its bits and the rest to nearest (2^-16 relative together; their sum is of the terms),
//     as in dense_kernel with four heads and more: the fp32 output is as exact as without groups (2-norm of the error, 2112
//     rows: 3.6e-6, and 6.7e-6 without, where the second term is cut off; 1.9e-7 with the fp32 weights that own rows of fewer heads have).
//     One term, 2^-8, is a third less to multiply, but made the fp32 output as coarse as the bf16 one: 32 sequences behind 32768 rows, 72
//     in three groups, 12 behind 131072 and 256 behind 16384 took 65, 170, 109 and 224 us with it, on one card in turn 72, 183, 112 and
//     280 with two.  The matrix cores bound groups of more than some 140 query rows a KV head.
#include <algorithm>
#include "hata_attn_core.h"
#include "hata_device.h"
#include "hata_internal.h"

namespace hata {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;

#define PREFIX_TILE 64       // rows that runs are cut by; what is left of the common rows is read by every sequence itself
#define PREFIX_MAX_SPLITS 256
#define PREFIX_LOOSE 56.f
#define PREFIX_LDS (4 * 64 * (HATA_D + 4) * 4)  // the waves' sums at the end; before, the ring of stages

struct PrefixArgs {
    const uint16_t *q, *K, *V;
    const int32_t *seq_len, *group_start, *shared_len;
    PrefixPlan* plan;
    float* part;
    PageView pv;
    int B, Hq, Hkv, G, L_cap, n_groups, own_teams, own_spare, own_run;  // of the launch behind: teams at once, with those to spare, and the fewest tiles of a run
    float scale_log2;
};

// ---- which workgroup does what ----
//
// Every workgroup works it out for itself: the groups' members, the rows they have in common, and the shortest run (in tiles) at
// which the launch's workgroups suffice, one per (group, KV head, tile of query rows, run).  The tiles of query rows of a run are
// neighbours on one XCD, whose L2 then serves all but the first of them.  The last workgroup writes the plan that the launch behind
// goes by.  (A workgroup more than there are compute units would have to wait for one.)  It has nothing else to do, unless the
// others' runs would be longer for that by more than the plan takes (5 us; a tile of rows takes 0.8 us for 64 query rows).
struct PrefixShare { int g, h, split, ns, qt, tiles, item, first, members, lead; };
struct PrefixGroups { int *start, *least, *count, *lead; };  // in LDS: first member [n + 1]; tiles in common, members that have rows, the first of them [n]

__device__ __forceinline__ PrefixGroups prefix_groups(const PrefixArgs& a, int* lds) {
    const int n = a.n_groups, tid = threadIdx.x;
    int* start = lds;
    int* least = start + n + 1;
    int* count = least + n;
    int* lead = count + n;
    int* shared = lead + n;
    const int own = a.seq_len[min(tid, a.B - 1)];  // (on its way with the groups')
    for (int i = tid; i <= n; i += 256) {
        start[i] = clampi(a.group_start[i], 0, a.B);
        if (i < n) { least[i] = 0x7fffffff; count[i] = 0; lead[i] = 0x7fffffff; shared[i] = a.shared_len[i]; }
    }
    __syncthreads();
    int falls = 0;
    for (int i = tid; i < n; i += 256) falls |= start[i] > start[i + 1];
    if (__syncthreads_or(falls)) {  // ascending, whatever the caller gave
        if (tid == 0)
            for (int i = 1; i <= n; ++i) start[i] = max(start[i], start[i - 1]);
        __syncthreads();
    }
    for (int b0 = 0; b0 < a.B; b0 += 256) {
        const int b = b0 + tid, L = b < a.B ? clampi(b0 ? a.seq_len[b] : own, 0, a.L_cap) : 0;
        int g = -1;
        if (L > 0 && b >= start[0] && b < start[n]) {
            int c = n;  // the last group that begins at b or before
            g = 0;
            while (c > 1) {
                const int h = c / 2;
                if (start[g + h] <= b) { g += h; c -= h; }
                else c = h;
            }
        }
        const unsigned long long some = __builtin_amdgcn_ballot_w64(g >= 0);
        if (!some) continue;
        const int l0 = __ffsll(some) - 1, g0 = __builtin_amdgcn_readlane(g, l0);
        if (__builtin_amdgcn_ballot_w64(g >= 0 && g != g0) == 0ull) {  // a wave of one group (lengths are below 2^24)
            const int low = (int)-wave_max64(g >= 0 ? -(float)L : HATA_NEG_INF);
            if ((tid & 63) == l0) {
                atomicMin(&least[g], low);
                atomicAdd(&count[g], __popcll(some));
                atomicMin(&lead[g], b);
            }
        } else if (g >= 0) {
            atomicMin(&least[g], L);
            atomicAdd(&count[g], 1);
            atomicMin(&lead[g], b);
        }
    }
    __syncthreads();
    for (int g = tid; g < n; g += 256) least[g] = count[g] >= 2 ? max(min(shared[g], least[g]), 0) / PREFIX_TILE : 0;
    __syncthreads();
    return PrefixGroups{start, least, count, lead};
}

// The run length, and through `each` the groups of every 64 (lane: group g, its tiles of query rows, its runs, its first item)
template <typename Each>
__device__ __forceinline__ void prefix_items(const PrefixArgs& a, const PrefixGroups& s, int mpt, int wgs, Each each) {
    const int n = a.n_groups, lane = threadIdx.x & 63;
    auto qtiles = [&](int g) { return g < n ? (s.start[g + 1] - s.start[g] + mpt - 1) / mpt : 0; };
    auto tiles = [&](int g) { return g < n ? s.least[g] : 0; };
    const int qt0 = qtiles(lane), tiles0 = tiles(lane);  // (all there is, mostly)
    float all = wave_sum64((float)qt0 * tiles0), longest = wave_max64((float)tiles0);
    for (int g0 = 64; g0 < n; g0 += 64) {
        all += wave_sum64((float)qtiles(g0 + lane) * tiles(g0 + lane));
        longest = fmaxf(longest, wave_max64((float)tiles(g0 + lane)));
    }
    auto splits = [](int t, int run) { return min((t + run - 1) / run, PREFIX_MAX_SPLITS); };
    int run = max(1, (int)ceilf(all * (float)a.Hkv / (float)wgs)), with_last = 0;
    for (;; run += max(1, run >> 4)) {
        uint32_t items = (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_scan((uint32_t)(qt0 * splits(tiles0, run))), 63);
        for (int g0 = 64; g0 < n; g0 += 64)
            items += (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_scan((uint32_t)(qtiles(g0 + lane) * splits(tiles(g0 + lane), run))), 63);
        items *= (uint32_t)a.Hkv;
        if (items == (uint32_t)wgs && !with_last) with_last = run;  // (the workgroup with the plan would have an item too)
        if (items < (uint32_t)wgs || run >= (int)longest) break;
    }
    if (with_last && (run - with_last) * mpt * a.G > 6 * 64) run = with_last;
    uint32_t base = 0;
    for (int g0 = 0; g0 < n; g0 += 64) {
        const int g = g0 + lane, qt = g0 ? qtiles(g) : qt0, ns = splits(g0 ? tiles(g) : tiles0, run);
        const uint32_t upto = wave_incl_scan((uint32_t)(a.Hkv * qt * ns));
        if (each(g, qt, ns, (int)(base + upto) - a.Hkv * qt * ns)) return;
        base += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    }
}

__device__ __forceinline__ bool prefix_share(const PrefixArgs& a, int mpt, int* lds, PrefixShare& w) {
    const int item = (int)((blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8);
    const PrefixGroups s = prefix_groups(a, lds);
    w.g = -1;
    prefix_items(a, s, mpt, gridDim.x, [&](int g, int qt, int ns, int base) {
        const unsigned long long here = __builtin_amdgcn_ballot_w64(item >= base && item < base + a.Hkv * qt * ns);
        if (!here) return false;
        const int l = __ffsll(here) - 1;
        w.g = __builtin_amdgcn_readlane(g, l);
        qt = __builtin_amdgcn_readlane(qt, l);
        ns = __builtin_amdgcn_readlane(ns, l);
        const int in = item - __builtin_amdgcn_readlane(base, l);
        w.ns = ns;
        w.item = item;
        w.qt = in % qt;
        w.split = in / qt % ns;
        w.h = in / (qt * ns);
        w.tiles = __builtin_amdgcn_readfirstlane(s.least[w.g]);
        w.lead = __builtin_amdgcn_readfirstlane(s.lead[w.g]);
        const int start = __builtin_amdgcn_readfirstlane(s.start[w.g]);
        w.first = start + w.qt * mpt;
        w.members = min(mpt, __builtin_amdgcn_readfirstlane(s.start[w.g + 1]) - w.first);
        return true;
    });
    __syncthreads();  // (the LDS is used anew)
    return w.g >= 0;
}

// The plan for the rows that are left to the sequences: where they begin, and runs of them for the teams of the launch behind -- the
// shortest run length (at least PREFIX_OWN_RUN tiles of 16 rows a wave) at which its teams suffice.
#define PREFIX_OWN_RUN 2
#define PREFIX_OWN_RUNS 256  // of a unit
__device__ __forceinline__ void prefix_plan(const PrefixArgs& a, int mpt, int* lds) {
    const int n = a.n_groups, tid = threadIdx.x, lane = tid & 63;
    const PrefixGroups s = prefix_groups(a, lds);
    int* rows = lds + 5 * n + 1;  // [B] behind the shared ones
    static_assert((5 * HATA_PREFIX_GROUPS + 1 + HATA_PREFIX_MAX_B) * 4 <= PREFIX_LDS, "room for the plan");
    for (int b = tid; b < a.B; b += 256) {
        const int L = clampi(a.seq_len[b], 0, a.L_cap);
        rows[b] = L;
        if (L == 0 || b < s.start[0] || b >= s.start[n]) a.plan[b] = PrefixPlan{0, 0, L, 0, 0, 0, 0, 1};
    }
    __syncthreads();
    prefix_items(a, s, mpt, gridDim.x, [&](int g, int qt, int ns, int base) {
        // (a wave's lanes have a group each; the four waves share its members)
        for (unsigned long long left = __builtin_amdgcn_ballot_w64(g < n); left; left &= left - 1) {
            const int l = __ffsll(left) - 1, gl = __builtin_amdgcn_readlane(g, l);
            const int qtl = __builtin_amdgcn_readlane(qt, l), nsl = __builtin_amdgcn_readlane(ns, l), at = __builtin_amdgcn_readlane(base, l);
            const int start = s.start[gl], first = s.least[gl] * PREFIX_TILE;
            for (int b = start + tid; b < s.start[gl + 1]; b += 256) {
                const int i = b - start, L = rows[b];
                if (L == 0) continue;
                rows[b] = L - first;
                a.plan[b] = PrefixPlan{0, 0, L - first, first, at + i / mpt, nsl, i % mpt * a.G, max(qtl, 1)};
            }
        }
        return false;
    });
    __syncthreads();
    auto tiles = [&](int b) { return b < a.B ? (max(rows[b], 1) + 15) / 16 : 0; };
    float all = 0.f, longest = 0.f;
    for (int b = lane; b < a.B; b += 64) {
        all += (float)tiles(b);
        longest = fmaxf(longest, (float)tiles(b));
    }
    all = wave_sum64(all);
    longest = wave_max64(longest);
    int run = 0;
    auto runs = [&](int b) { return (uint32_t)min((tiles(b) + run - 1) / run, PREFIX_OWN_RUNS); };
    auto search = [&](int teams) {
        run = max(a.own_run, (int)ceilf(all * (float)a.Hkv / (float)teams));
        if (a.B * a.Hkv >= teams) run = max(run, (int)longest);  // (one a unit)
        for (;; run += max(1, run >> 4)) {
            float n = 0.f;  // (below 2^24)
            for (int b = lane; b < a.B; b += 64) n += (float)runs(b);
            if (wave_sum64(n) * (float)a.Hkv <= (float)teams || run >= (int)longest) return run;
        }
    };
    const int spare = search(a.own_spare), at_once = search(a.own_teams);
    if (at_once > 2 * spare + 8 * a.own_run) run = spare;  // (a second round of workgroups)
    uint32_t start = 0;
    for (int b0 = 0; b0 < a.B; b0 += 64) {
        const int b = b0 + lane;
        const uint32_t r = runs(b), upto = wave_incl_scan(r);
        if (tid < 64 && b < a.B) {
            a.plan[b].start = (int)((start + upto - r) * a.Hkv);
            a.plan[b].runs = (int)r;
        }
        start += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    }
    __syncthreads();  // (the LDS is used anew)
}

// 16-byte piece c of row r of a stage is at slot c ^ prefix_swizzle(r): 16 rows of one piece, and four rows of four pieces, are in
// 16 different slots, so that neither product's reads have bank conflicts
__device__ __forceinline__ int prefix_swizzle(int r) { return (r & 3) << 2 | (r >> 2 & 3); }

// (fmaxf alone costs an instruction more for each operand, to quiet a NaN that is dropped anyway)
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// Two weights as two bf16 terms each, of one sign: the upper half, and what is left of it rounded to nearest
__device__ __forceinline__ uint32_t prefix_high(float x, float y) {
    return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
}
__device__ __forceinline__ uint32_t prefix_low(float x, float y) {
    f32x2_t e;
    e[0] = x - __uint_as_float(__float_as_uint(x) & 0xffff0000u);
    e[1] = y - __uint_as_float(__float_as_uint(y) & 0xffff0000u);
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(e, bf16x2_t));
}

template <int N>
__device__ __forceinline__ void prefix_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// WQ: waves with query rows of their own.  A stage is 4 / WQ parts (one per wave with the same query rows) of PART rows, K and V.
template <int WQ>
__global__ __launch_bounds__(256, 1) void prefix_kernel(const PrefixArgs a) {
    constexpr int WK = 4 / WQ, PART = WQ == 4 ? 64 : 32, STAGE = WK * PART, SUBS = PART / 32;
    constexpr int NBUF = 256 / STAGE;                                // stages in LDS: 128 KB
    constexpr int BLOCKS = PART / WQ / 16;                           // blocks of 16 rows a wave requests of a stage, K and V
    constexpr int M = 64 * WQ;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wq = wave % WQ, wk = wave / WQ, n = lane & 31, half = lane >> 5;
    if (blockIdx.x == gridDim.x - 1) prefix_plan(a, M / a.G, reinterpret_cast<int*>(smem));
    PrefixShare w;
    if (!prefix_share(a, M / a.G, reinterpret_cast<int*>(smem), w)) return;
    const int G = a.G, rows = w.members * G;
    // rows of this workgroup, in tiles of 64; of a stage of 128 that reaches over the end the waves behind it have nothing to do
    const int t0 = (int)((int64_t)w.tiles * w.split / w.ns), t1 = (int)((int64_t)w.tiles * (w.split + 1) / w.ns);
    const int k0 = t0 * PREFIX_TILE, k1 = t1 * PREFIX_TILE, stages = (k1 - k0 + STAGE - 1) / STAGE;

    // operands of the query rows: row 64 wq + 32 t + n, channels 16 s + 8 half ..
    uint4 qb[2][8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int r = min(64 * wq + 32 * t + n, rows - 1);
        const uint16_t* qr = a.q + ((int64_t)(w.first + r / G) * a.Hq + w.h * G + r % G) * HATA_D + 8 * half;
#pragma unroll
        for (int s = 0; s < 8; ++s) qb[t][s] = *reinterpret_cast<const uint4*>(qr + 16 * s);
    }
    const float scale = fabsf(a.scale_log2);
    if (a.scale_log2 < 0.f) {  // (the maximum of the products is that of the scores then)
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                qb[t][s].x ^= 0x80008000u; qb[t][s].y ^= 0x80008000u;
                qb[t][s].z ^= 0x80008000u; qb[t][s].w ^= 0x80008000u;
            }
    }

    const uint32_t ring = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)smem);
    // Page numbers by scalar loads, a stage ahead: a wait for a vector load is one for every request in flight
    const auto table = (const __attribute__((address_space(4))) int32_t*)(uintptr_t)(a.pv.table + (int64_t)w.lead * a.pv.max_blocks);
    int pages[BLOCKS];
    auto first_row = [&](int s, int j) { return min(k0 + s * STAGE + wk * PART + (wq * BLOCKS + j) * 16, k1 - 16); };
    auto look_up = [&](int s) {
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) pages[j] = table[first_row(s, j) >> a.pv.shift];
    };
    look_up(0);
    // this wave's rows of a stage: PART wk + 16 BLOCKS wq + 16 j ..; lane l of an instruction fetches, of row 4 i + l / 16 of a block,
    // the piece that belongs at slot l % 16
    uint32_t off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) off[i] = (4 * i + (lane >> 4)) * 256 + ((lane & 15) ^ (lane >> 4 << 2 | i)) * 16;
    // (written as instructions: behind the compiler's builtin for it, every LDS read waits for all requests.  nt where the rows are read
    // by one tile of query rows, mostly: 12 sequences behind 131072 rows 119 -> 108 us, 32 behind 32768 68 -> 63; with eight tiles
    // it is the same, and slower where the caches hold the rows already)
    auto fetch = [&](uint32_t dst, uint32_t o, const uint16_t* p) {
        if constexpr (WQ <= 2)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(dst), "v"(o), "s"(p) : "memory", "m0");
        else
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(o), "s"(p) : "memory", "m0");
    };
    auto request = [&](int s) {
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) {
            const int row = first_row(s, j), page = clampi(pages[j], 0, a.pv.n_pages - 1);
            const int64_t at = ((((int64_t)page * a.Hkv + w.h) << a.pv.shift) + (row & ((1 << a.pv.shift) - 1))) * HATA_D;
            const uint32_t dst = ring + (uint32_t)((s % NBUF) * STAGE * 512 + (wk * PART + (wq * BLOCKS + j) * 16) * 256);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                fetch(dst + i * 1024, off[i], a.K + at);
                fetch(dst + STAGE * 256 + i * 1024, off[i], a.V + at);
            }
        }
        look_up(s + 1);
    };
    // The sums and the query rows live in the accumulation registers, where the matrix instructions take them from, the scores in the
    // others; said at every turn, or the compiler moves the sums to and fro
    f32x16_t acc[2][4];
    float m[2] = {HATA_NEG_INF, HATA_NEG_INF}, sub[2] = {0.f, 0.f}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][c][i] = 0.f;
    auto pin = [&]() {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) asm volatile("" : "+a"(acc[t][c]));
    };
    // K operand: row n, piece 2 s + half.  V operand: rows 16 x + 4 half + 8 y + (lane % 16) / 4, channels 32 c + lane's 16 and the
    // four of lane % 4
    const uint32_t k_at = n * 256 + ((half ^ prefix_swizzle(n)) << 4);
    const int v_row = 4 * half + (lane & 15) / 4, v_piece = (lane >> 4 & 1) * 2 + ((lane & 3) >> 1);

    auto products = [&](const char* kt, f32x16_t (&sc)[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[t][i] = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(kt + (k_at ^ (k << 5))));
#pragma unroll
            for (int t = 0; t < 2; ++t)
                sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, __builtin_bit_cast(bf16x8_t, qb[t][k]), sc[t], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) asm volatile("" : "+v"(sc[t]));
    };
    auto highest = [&](const f32x16_t (&sc)[2], float (&top)[2]) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            top[t] = sc[t][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top[t] = fmaxf(top[t], sc[t][i]);
            top[t] *= scale;
        }
    };
    // the references, where the highest scores pass one
    auto follow = [&](const float (&top)[2]) {
        if (__builtin_amdgcn_ballot_w64(top[0] > m[0] || top[1] > m[1]) != 0ull) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float x, y;
                swap32(top[t], x, y);
                const float high = fmaxf(x, y), to = high > m[t] ? high + PREFIX_LOOSE : m[t];  // (both halves' rows)
                const float f = m[t] == HATA_NEG_INF ? (to == HATA_NEG_INF ? 1.f : 0.f) : fast_exp2(m[t] - to);
                l[t] *= f;
#pragma unroll
                for (int c = 0; c < 4; ++c) acc[t][c] *= f;
                m[t] = to;
                sub[t] = to == HATA_NEG_INF ? 0.f : to;
            }
            pin();
        }
    };
    // (p: the terms of two rows' weights, [high or low][query row][two rows])
    auto weights = [&](const f32x16_t (&sc)[2], uint32_t (&p)[2][2][8]) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = fast_exp2(fmaf(sc[t][2 * i], scale, -sub[t])), y = fast_exp2(fmaf(sc[t][2 * i + 1], scale, -sub[t]));
                p[0][t][i] = prefix_high(x, y);
                p[1][t][i] = prefix_low(x, y);
                l[t] = dot2_bf16(p[1][t][i], 0x3f803f80u, dot2_bf16(p[0][t][i], 0x3f803f80u, l[t]));
            }
    };
    auto values = [&](const char* vt, const uint32_t (&p)[2][2][8]) {
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint2 v[2];
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const int r = 16 * x + 8 * y + v_row;
                    const s16x4_t av = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)const_cast<char*>(
                        vt + r * 256 + (((4 * c + v_piece) ^ prefix_swizzle(r)) << 4) + (lane & 1) * 8));
                    v[y] = __builtin_bit_cast(uint2, av);
                }
                const bf16x8_t vf = __builtin_bit_cast(bf16x8_t, make_uint4(v[0].x, v[0].y, v[1].x, v[1].y));
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int t = 0; t < 2; ++t)
                        acc[t][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            vf, __builtin_bit_cast(bf16x8_t, make_uint4(p[k][t][4 * x], p[k][t][4 * x + 1], p[k][t][4 * x + 2], p[k][t][4 * x + 3])), acc[t][c], 0, 0, 0);
            }
    };
    auto at_stage = [&](int s) { return (const char*)smem + (s % NBUF) * STAGE * 512 + wk * PART * 256; };  // K; V is STAGE * 256 bytes behind

    // (the wait for the query rows is one for every request so far: the first stage's only)
    request(0);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int s = 0; s < 8; ++s)  // (used here, so that the wait for these loads is not in the loop)
            asm volatile("" : "+a"(qb[t][s].x), "+a"(qb[t][s].y), "+a"(qb[t][s].z), "+a"(qb[t][s].w));
    pin();
    // (with several query waves a stage behind the last one is the last rows once more: as many requests are outstanding everywhere)
    for (int s = 1; s < NBUF - (WQ > 1); ++s)
        if (WQ > 1 || s < stages) request(s);
    if constexpr (WQ == 1) {
        // rows of this wave alone: nothing is waited for but its own requests
        for (int s = 0; s < stages; ++s) {
            if (s + 1 < stages) prefix_wait<BLOCKS * 8>();
            else prefix_wait<0>();
            if (k0 + s * STAGE + wk * PART < k1) {
                f32x16_t sc[2];
                uint32_t p[2][2][8];
                float top[2];
                products(at_stage(s), sc);
                highest(sc, top);
                follow(top);
                weights(sc, p);
                values(at_stage(s) + STAGE * 256, p);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // every read of this stage has returned
            if (s + NBUF < stages) request(s + NBUF);
            pin();
        }
    } else {
        // The products of the next 32 rows stand beside the weights of these, and their maxima beside these rows' second product:
        // matrix cores and vector ALU at work together, in one straight piece of code (what is computed behind the last rows is
        // of stale LDS and not used)
        f32x16_t sc[2], next[2];
        float top[2];
        prefix_wait<(NBUF - 2) * 8>();
        __syncthreads();
        products(at_stage(0), sc);
        highest(sc, top);
        for (int s = 0; s < stages; ++s) {
#pragma unroll
            for (int i = 0; i < SUBS; ++i) {
                uint32_t p[2][2][4];  // [turn and turn][query row][two rows]
                follow(top);
                // stage s + 1 is there once only the one behind it is outstanding; everybody is done with stage s - 1, whose place
                // the requests of this turn fill
                static_assert(BLOCKS == 1, "eight requests a stage");
                const bool turn = i + 1 == SUBS;
                uint32_t dst = 0;
                const uint16_t *k_from = nullptr, *v_from = nullptr;
                if (turn) {
                    prefix_wait<(NBUF - 3) * 8>();
                    __syncthreads();
                    const int row = first_row(s + NBUF - 1, 0), page = clampi(pages[0], 0, a.pv.n_pages - 1);
                    const int64_t at = ((((int64_t)page * a.Hkv + w.h) << a.pv.shift) + (row & ((1 << a.pv.shift) - 1))) * HATA_D;
                    dst = ring + (uint32_t)(((s + NBUF - 1) % NBUF) * STAGE * 512 + (wk * PART + wq * 16) * 256);
                    k_from = a.K + at;
                    v_from = a.V + at;
                    look_up(s + NBUF);
                }
                // (left to itself the compiler puts the matrix instructions one behind the other)
                const char* kt = i + 1 < SUBS ? at_stage(s) + (i + 1) * 32 * 256 : at_stage(s + 1);
                const char* vt = at_stage(s) + STAGE * 256 + i * 32 * 256;
                auto k_piece = [&](int k) { return __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(kt + (k_at ^ (k << 5)))); };
                bf16x8_t kf[3] = {k_piece(0), k_piece(1), k_piece(2)};
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int j = 0; j < 16; ++j) next[t][j] = 0.f;
                // (arguments, then weights, in the scores' place)
                auto argument = [&](int j) {
                    sc[j / 8][2 * (j % 8)] = fmaf(sc[j / 8][2 * (j % 8)], scale, -sub[j / 8]);
                    sc[j / 8][2 * (j % 8) + 1] = fmaf(sc[j / 8][2 * (j % 8) + 1], scale, -sub[j / 8]);
                };
                auto power = [&](int j) {
                    sc[j / 8][2 * (j % 8)] = fast_exp2(sc[j / 8][2 * (j % 8)]);
                    sc[j / 8][2 * (j % 8) + 1] = fast_exp2(sc[j / 8][2 * (j % 8) + 1]);
                };
                // group g of the second product: term g % 2 of the weights of rows 16 (g / 2) ..; two rows' of query row t
                auto term = [&](int g, int t, int i) {
                    const float x = sc[t][8 * (g / 2) + 2 * i], y = sc[t][8 * (g / 2) + 2 * i + 1];
                    p[g % 2][t][i] = g % 2 ? prefix_low(x, y) : prefix_high(x, y);
                    l[t] = dot2_bf16(p[g % 2][t][i], 0x3f803f80u, l[t]);
                };
                argument(0);
                power(0);
                argument(1);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    next[j % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[j / 2 % 3], __builtin_bit_cast(bf16x8_t, qb[j % 2][j / 2]), next[j % 2], 0, 0, 0);
                    if (j % 2 == 1 && j / 2 + 3 < 8) kf[j / 2 % 3] = k_piece(j / 2 + 3);
                    if (j + 1 < 16) power(j + 1);
                    if (j + 2 < 16) argument(j + 2);
                    if (j % 8 < 4) term(0, j / 8, j % 8);
                    if (turn && j % 2 == 0) fetch(dst + (j / 4) * 1024 + (j / 2 % 2) * STAGE * 256, off[j / 4], j / 2 % 2 ? v_from : k_from);
                    __builtin_amdgcn_sched_barrier(0);
                }
                auto v_piece_at = [&](int j) {  // channels 32 (j % 4) of rows 16 (j / 8) ..
                    uint2 v[2];
#pragma unroll
                    for (int y = 0; y < 2; ++y) {
                        const int r = 16 * (j / 8) + 8 * y + v_row;
                        v[y] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4_t*)const_cast<char*>(
                            vt + r * 256 + (((4 * (j % 4) + v_piece) ^ prefix_swizzle(r)) << 4) + (lane & 1) * 8)));
                    }
                    return __builtin_bit_cast(bf16x8_t, make_uint4(v[0].x, v[0].y, v[1].x, v[1].y));
                };
                bf16x8_t vf[3] = {v_piece_at(0), v_piece_at(1), v_piece_at(2)};
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const int g = j / 8, t = j % 2, c = j / 2 % 4, i = j / 2 % 4;
                    const auto& w = p[g % 2][t];
                    acc[t][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        vf[j / 2 % 3], __builtin_bit_cast(bf16x8_t, make_uint4(w[0], w[1], w[2], w[3])), acc[t][c], 0, 0, 0);
                    if (j % 2 == 1 && j / 2 + 3 < 16) vf[j / 2 % 3] = v_piece_at(j / 2 + 3);
                    if (g < 3) term(g + 1, t, i);
                    if (g % 2) {  // (the groups with less to do beside them)
                        const int k = g / 2;
                        if (j % 8 == 0) {
                            asm volatile("" : "+v"(next[k]));
                            top[k] = fmaxf(next[k][0], next[k][1]);
                        } else {
                            top[k] = max3(top[k], next[k][2 * (j % 8)], next[k][2 * (j % 8) + 1]);
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                top[0] *= scale;
                top[1] *= scale;
#pragma unroll
                for (int t = 0; t < 2; ++t) sc[t] = next[t];
                pin();
            }
        }
    }

    // ---- the waves' sums, joined where they have the same query rows ----
    prefix_wait<0>();
    __syncthreads();  // the ring is no longer read
    float* s_acc = reinterpret_cast<float*>(smem);  // [wave][64][HATA_D + 4]
    __shared__ float s_m[4][64], s_l[4][64];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        float x, y;
        swap32(l[t], x, y);
        l[t] = x + y;
        if (half == 0) { s_m[wave][32 * t + n] = m[t]; s_l[wave][32 * t + n] = l[t]; }
    }
    float top[2] = {m[0], m[1]}, total[2] = {l[0], l[1]};
    if constexpr (WK > 1) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
            for (int k = 0; k < WK; ++k) top[t] = fmaxf(top[t], s_m[wq + k * WQ][32 * t + n]);
            total[t] = 0.f;
#pragma unroll
            for (int k = 0; k < WK; ++k) {
                const float mk = s_m[wq + k * WQ][32 * t + n];
                total[t] = fmaf(mk == HATA_NEG_INF ? 1.f : fast_exp2(mk - top[t]), s_l[wq + k * WQ][32 * t + n], total[t]);
            }
            const float f = m[t] == HATA_NEG_INF ? 1.f : fast_exp2(m[t] - top[t]);  // (sums without a score are zero)
#pragma unroll
            for (int c = 0; c < 4; ++c) acc[t][c] *= f;
        }
    }
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)  // acc[t][c][4 i + j]: channel 32 c + 8 i + 4 half + j of query row 32 t + n
                *reinterpret_cast<float4*>(&s_acc[(wave * 64 + 32 * t + n) * (HATA_D + 4) + 32 * c + 8 * i + 4 * half]) =
                    make_float4(acc[t][c][4 * i], acc[t][c][4 * i + 1], acc[t][c][4 * i + 2], acc[t][c][4 * i + 3]);
    __syncthreads();
    float* out = a.part + (int64_t)w.item * (M * (HATA_D + 2));
    if (wk == 0 && half == 0) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
            if (64 * wq + 32 * t + n < rows)
                *reinterpret_cast<float2*>(out + M * HATA_D + 2 * (64 * wq + 32 * t + n)) = make_float2(top[t], total[t]);
    }
    // eight rows a turn, four turns together
    const int r8 = tid / 32, c4 = tid % 32 * 4;
    for (int i0 = 0; i0 < rows; i0 += 32) {
        float4 o[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = i0 + 8 * j + r8;  // (rows up to M lie in LDS)
            o[j] = *reinterpret_cast<const float4*>(&s_acc[(r / 64 * 64 + r % 64) * (HATA_D + 4) + c4]);
#pragma unroll
            for (int k = 1; k < WK; ++k) {
                const float4 v = *reinterpret_cast<const float4*>(&s_acc[((r / 64 + k * WQ) * 64 + r % 64) * (HATA_D + 4) + c4]);
                o[j].x += v.x; o[j].y += v.y; o[j].z += v.z; o[j].w += v.w;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i0 + 8 * j + r8 < rows) *reinterpret_cast<float4*>(out + (i0 + 8 * j + r8) * HATA_D + c4) = o[j];
    }
}

// Query rows of a workgroup (waves with rows of their own), 64, 128 or 256, from the mean of the groups.  A tile larger than
// the group leaves waves without query rows, where a smaller one's go over different rows; a larger one reads the rows less often.
// us of a call with 64 / 128 / 256, one group behind 32768 rows and up to 200 of their own, eight KV heads, groups of four: 64 query rows
// 48.2 / 55.9 / 77.0, 96 59.4 / 57.0 / 75.5, 128 60.0 / 58.4 / 75.9, 192 77.3 / 81.1 / 82.8, 256 92.4 / 85.3 / 88.0, 384 127 / 114 / 126,
// 448 149 / 135 / 131, 512 155 / 138 / 134; behind 4096 rows 64 30.1 / 30.9 / 33.2, 128 31.1 / 34.9 / 36.1, 256 38.3 / 39.8 / 45.0, 512
// 55.2 / 51.5 / 54.6 (how long the shared rows are is not known on the host).  The mean is of all sequences, those in no group too, which
// is what the host knows: with eight sequences behind 32768 rows and 150 alone, of 1024 rows each, it gives 256 to a group of 32 query rows,
// 171 us (148 with 64, 208 without groups).
#define PREFIX_ROWS_64 64
#define PREFIX_ROWS_128 448
static int prefix_waves(int64_t rows_per_group) { return rows_per_group <= PREFIX_ROWS_64 ? 1 : rows_per_group <= PREFIX_ROWS_128 ? 2 : 4; }

// Workgroups of a launch: one per compute unit, or as many as the (tile of query rows, KV head) of groups with two members and more need
static int64_t prefix_wgs(int B, int Hkv, int G, int n_groups, int waves) {
    const int mpt = 64 * waves / G;
    const int64_t tiles = (B + (int64_t)std::min(n_groups, B / 2) * (mpt - 1)) / mpt * Hkv;
    return std::max((int64_t)256, (tiles + 255) / 256 * 256);
}

size_t prefix_part_floats(int B, int Hkv, int G) {
    if (B < 2) return 0;
    B = std::min(B, HATA_PREFIX_MAX_B);
    size_t most = 0;
    for (int waves = 1; waves <= 4; waves *= 2) {
        // the most groups that go by so many waves
        const int64_t above = waves == 1 ? 0 : waves == 2 ? PREFIX_ROWS_64 : PREFIX_ROWS_128;
        const int64_t groups = std::min((int64_t)std::min(B, HATA_PREFIX_GROUPS), above ? ((int64_t)B * G - 1) / above : (int64_t)B);
        if (groups < 1) continue;
        most = std::max(most, (size_t)prefix_wgs(B, Hkv, G, (int)groups, waves) * 64 * waves * (HATA_D + 2));
    }
    return most;
}

hipError_t prepare_prefix() {
    for (const void* fn : {(const void*)prefix_kernel<1>, (const void*)prefix_kernel<2>, (const void*)prefix_kernel<4>}) {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, PREFIX_LDS);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_prefix(const hata_ctx* c, const void* q, const void* K, const void* V, const PageView& pages, const int32_t* seq_len, int B,
                         const int32_t* group_start, const int32_t* shared_len, int n_groups, float sm_scale, int* part_rows, hipStream_t s) {
    const hata_config& f = c->cfg;
    PrefixArgs a;
    a.q = (const uint16_t*)q; a.K = (const uint16_t*)K; a.V = (const uint16_t*)V;
    a.seq_len = seq_len; a.group_start = group_start; a.shared_len = shared_len;
    a.plan = c->prefix_plan;
    const int team = dense_own_team(B, f.Hkv);
    a.own_teams = dense_own_wgs(B, f.Hkv, false) * 8 / team;
    a.own_spare = dense_own_wgs(B, f.Hkv, true) * 8 / team;
    a.own_run = PREFIX_OWN_RUN * team;
    a.part = c->prefix_part;
    a.pv = pages;
    a.B = B; a.Hq = f.Hq; a.Hkv = f.Hkv; a.G = c->G;
    a.L_cap = (int)std::min((int64_t)f.L_cap, (int64_t)pages.max_blocks << pages.shift);
    a.n_groups = n_groups;
    a.scale_log2 = sm_scale * 1.4426950408889634f;
    const int waves = prefix_waves(((int64_t)B * c->G + n_groups - 1) / n_groups);
    *part_rows = 64 * waves;
    const dim3 grid((unsigned)prefix_wgs(B, f.Hkv, c->G, n_groups, waves));
    hipLaunchKernelGGL((waves == 1 ? prefix_kernel<1> : waves == 2 ? prefix_kernel<2> : prefix_kernel<4>), grid, dim3(256), PREFIX_LDS, s, a);
    return hipGetLastError();
}

}  // namespace hata
