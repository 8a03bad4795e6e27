// Decode attention over rows that a group of sequences has in common (Eq. 1 of the paper, block tables): read once for all of
// them.  For the query rows i of a group's members (member by member, the G heads of a KV head side by side) and a run of the
// common rows,
//   l_i = sum_n 2^(s_in - m_i),  o_i = sum_n 2^(s_in - m_i) V_n,   s_in = scale log2(e) q_i . K_n,  m_i >= max_n s_in,
// which dense_kernel joins with the sequences' own rows.  How a workgroup goes over its rows: hata_shared_rows.h.
#include <algorithm>
#include "hata_attn_core.h"
#include "hata_device.h"
#include "hata_internal.h"
#include "hata_shared_rows.h"

namespace hata {

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

template <int WQ>
__global__ __launch_bounds__(256, 1) void prefix_kernel(const PrefixArgs a) {
    constexpr int M = 64 * WQ;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    if (blockIdx.x == gridDim.x - 1) prefix_plan(a, M / a.G, reinterpret_cast<int*>(smem));
    PrefixShare w;
    if (!prefix_share(a, M / a.G, reinterpret_cast<int*>(smem), w)) return;
    shared_rows<WQ, 2, false>(a, w, smem);
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
