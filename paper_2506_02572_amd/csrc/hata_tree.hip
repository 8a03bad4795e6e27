// Attention of drafted tokens on block tables (hata_dense_tree_paged), and the rows of the accepted ones (hata_keep_rows).
//
// Token i of a sequence of `base` committed rows:  o_i = sum_n w_in V_n / sum_n w_in,  w_in = exp(scale q_i . K_n), over n < base and those
// drafted rows that i sees.  All tokens read the committed rows, so the tokens and the G heads of a KV head are the query rows of one
// matrix (hata_shared_rows.h), the rows are read once for up to 256 of them, and the mask costs only in the tiles that have drafted rows:
// there a score that is not seen becomes -inf in its register.  Bound by the bytes up to some 100 query rows, by the products behind
// that; they add on this device, and the products count 1.5 times, for the weights' second term.  32 sequences of 8192 rows and eight KV
// heads, G = 4, us with 1, 8, 16, 32 and 64 tokens each: 171, 170, 196, 295 and 491 (the rows alone, at 6.1 TB/s: 176).  A token
// and head at a time (the first form) 22400 us for what takes 252 here: 16 sequences of up to 16384 rows, the last up to 33 of them
// drafted, eight KV heads, G = 8.
// Why two terms: they leave the fp32 output 3e-6 to 5e-6 off (2-norm; normally distributed values, 300 to 32768 rows, any G; 3e-7 to 1.7e-6 with
// weights in fp32), which the bf16 output, rounded by 1.6e-3, does not show: with scores of tens, as outlier channels make them, 2 sequences of
// 131072 rows and 48 tokens are 1.60513e-3 off with either, 32 of 8192 rows and 64 tokens 1.53323e-3; 0.2 to 0.3 % of the values differ by
// a rounding, and in 42 to 50 % of those this one is the nearer.  (The fp32 outputs are 2.2e-6 and 1.9e-6 off there, and 2.7e-6 and 1.8e-6 with weights in
// fp32: the scores' own roundings.)  A third term would be a third more to multiply.
#include <algorithm>
#include "hata_attn_core.h"
#include "hata_device.h"
#include "hata_internal.h"
#include "hata_shared_rows.h"

namespace hata {

// Row n of sequence b and KV head h in the pools, in rows of HATA_D values
__device__ __forceinline__ int pool_row(const PageView& pv, int b, int n, int h, int Hkv) {
    const int page = clampi(pv.table[(int64_t)b * pv.max_blocks + (n >> pv.shift)], 0, pv.n_pages - 1);
    return ((page * Hkv + h) << pv.shift) + (n & ((1 << pv.shift) - 1));
}

// ---- which workgroup does what ----
//
// A unit is a KV head of a tile of a sequence's tokens (TREE_ROWS / G of them at most), and costs tree_start and for every tile of rows
// tree_weight.  All units, one behind the other, are cut into as many equal pieces as there are workgroups, wherever that
// falls; a workgroup goes through what lies in its piece.  Of these at most its first and its last one share a unit with
// other workgroups: they leave partial results (2 i, or 2 i + 1 where the unit begins in workgroup i), and the workgroup with the unit's
// first rows a record for the second launch.  A few units are cut into whole pieces each, of the shortest run of tiles at which the
// workgroups suffice.  Every workgroup works its share out from the lengths.
#define TREE_ROWS 256
#define TREE_WGS 256
#define TREE_LEAST 35   // what a piece costs at least: the largest weight (or, of 32 query rows, a turn of four waves)
#define TREE_LEAST_SMALL 16
#define TREE_WHOLE 64   // up to so many units no workgroup has parts of two
struct TreeRun { int members, t0, t1, h, first, lead, item, base, end, draft0; bool final; };
struct TreeSequence { int t0, n, base, end; };

__device__ __forceinline__ TreeSequence tree_sequence(const TreeArgs& a, int b) {
    TreeSequence q = {0, 0, 0, 0};
    if (b >= a.B) return q;
    q.t0 = clampi(a.token_start[b], 0, a.n_tokens);
    q.n = clampi(clampi(a.token_start[b + 1], 0, a.n_tokens) - q.t0, 0, a.max_draft);
    const int L = clampi(a.seq_len[b], 0, a.L_cap);
    q.base = clampi(a.base[b], 0, L);
    q.end = min(L, q.base + q.n);
    return q;
}
// Tenths of a microsecond: of a tile of rows, with 32, 64, 128 and 256 query rows, and of a unit beside its rows (measured in ragged batches)
__device__ __forceinline__ int tree_weight(int rows) { return rows <= 32 ? 8 : rows <= 64 ? 12 : rows <= 128 ? 21 : 35; }
// (where the units are fewer than the workgroups they are cut anyway, and every part has its own beginning)
__device__ __forceinline__ int tree_start(int weight, int units) { return (weight == 8 ? 70 : 130) * min(units, TREE_WGS) / TREE_WGS; }
struct TreeCosts {
    int tiles, qt, full, last, units;  // weights of a tile of TREE_ROWS query rows and of the last one
    __device__ __forceinline__ TreeCosts(const TreeSequence& q, int G, int all_units) : units(all_units) {
        const int mpt = TREE_ROWS / G;
        tiles = max(1, (q.end + PREFIX_TILE - 1) / PREFIX_TILE);
        qt = (q.n + mpt - 1) / mpt;
        full = tree_weight(TREE_ROWS);
        last = tree_weight((q.n - (qt - 1) * mpt) * G);
    }
    __device__ __forceinline__ int64_t unit(int weight) const { return tree_start(weight, units) + (int64_t)tiles * weight; }
    __device__ __forceinline__ int64_t head() const { return qt ? (qt - 1) * unit(full) + unit(last) : 0; }
    // the tile of rows at x of a unit
    __device__ __forceinline__ int tile_at(int64_t x, int weight) const {
        return (int)((uint32_t)max((int)x - tree_start(weight, units), 0) / (uint32_t)weight);
    }
};

// x / d of numbers that are not negative, mostly below 2^32
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t d) {
    if (((uint64_t)x | (uint64_t)d) >> 32) return x / d;
    return (uint32_t)x / (uint32_t)d;
}

struct TreeShare {
    int64_t pre[257];  // what lies in front of every thread's sequences
    int64_t at;        // the sequence that the next unit belongs to, and what lies in front of it
    int b;
    TreeSequence q;
    float tiles[4];
    uint32_t seen[TREE_ROWS * SEEN_WORDS];
    int row[TREE_ROWS], member[TREE_ROWS];  // of DraftTables
};

// Which drafted rows the tokens of this workgroup see
__device__ __forceinline__ void tree_seen(const TreeArgs& a, const TreeRun& w, uint32_t* seen) {
    auto below = [](int n) { return n >= 32 ? ~0u : n <= 0 ? 0u : (1u << n) - 1; };
    for (int e = threadIdx.x; e < w.members * SEEN_WORDS; e += 256) {
        const int i = e / SEEN_WORDS, k = e % SEEN_WORDS;
        uint32_t bits = 0;
        if (k < 8) bits = !a.mask ? below(w.draft0 + i + 1 - 32 * k) : k < a.words ? a.mask[(int64_t)(w.first + i) * a.words + k] : 0u;
        seen[e] = bits & below(w.end - w.base - 32 * k);
    }
}

// (The code in front of the rows runs once, out of a cold instruction cache: what a few sequences do not need stands apart.)
template <bool SMALL>
__global__ __launch_bounds__(256, 1) void tree_kernel(const TreeArgs a) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ TreeShare s;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wg = (int)((blockIdx.x % 8) * (TREE_WGS / 8) + blockIdx.x / 8), G = a.G, mpt = TREE_ROWS / G;
    constexpr int LEAST = SMALL ? TREE_LEAST_SMALL : TREE_LEAST;
    // every thread's sequences (of up to 64 every wave looks at all), and all units
    const bool few = a.B <= 64;
    const int per = few ? 1 : (a.B + 255) / 256, b0 = few ? lane : tid * per;
    const TreeSequence own = tree_sequence(a, b0);
    int units;
    {
        float n = (float)((own.n + mpt - 1) / mpt);
        for (int b = b0 + 1; b < b0 + per; ++b) n += (float)((tree_sequence(a, b).n + mpt - 1) / mpt);
        n = wave_sum64(n);
        if (!few) {
            if (lane == 0) s.tiles[wave] = n;
            __syncthreads();
            n = s.tiles[0] + s.tiles[1] + s.tiles[2] + s.tiles[3];
        }
        units = a.Hkv * (int)fminf(n, (float)TREE_WGS);  // (more do not matter)
    }
    {
        const int member = (int)(((float)tid + 0.5f) * __builtin_amdgcn_rcpf((float)G));
        s.member[tid] = member;
        s.row[tid] = member * a.Hq + tid - member * G;
    }
    const DraftTables tables = {s.seen, s.row, s.member};
    TreeRun w;
    TreeSplit split = {-1, 0, 0, 0};  // the unit that begins here and goes on elsewhere
    auto place = [&](const TreeSequence& q, int b, int h, int tile, int t0, int t1, int tiles) {
        auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };  // (as it is: said to the compiler)
        w.t0 = same(t0);
        w.t1 = same(t1);
        w.h = same(h);
        w.lead = same(b);
        w.base = same(q.base);
        w.end = same(q.end);
        w.draft0 = same(tile) * mpt;
        w.first = same(q.t0) + w.draft0;
        w.members = min(mpt, same(q.n) - w.draft0);
        w.final = w.t0 == 0 && w.t1 == tiles;
        w.item = 2 * wg + (w.t0 == 0 ? 1 : 0);
    };
    const bool whole = few && units <= TREE_WHOLE;
    int64_t pos = 0, p0 = 0, p1 = 0, total = 0, u0 = 0;
    int pieces = 1, h = 0, tile = 0, b = 0;
    TreeSequence q = {0, 0, 0, 0};
    bool again = false;
    if (whole) {
        const TreeCosts c(own, G, 0);
        const int full = c.tiles * c.full, last = c.tiles * c.last;
        const float all = wave_sum64(c.qt ? (float)(c.qt - 1) * full + last : 0.f) * a.Hkv;
        int kf, kl, mine, upto;  // pieces of a unit, and all of a sequence
        for (int run = max(LEAST, (int)ceilf(all / TREE_WGS));; run += max(1, run >> 4)) {
            kl = min((int)((uint32_t)(last + run - 1) / (uint32_t)run), c.tiles);
            kf = c.qt > 1 ? min((int)((uint32_t)(full + run - 1) / (uint32_t)run), c.tiles) : kl;
            mine = c.qt ? a.Hkv * ((c.qt - 1) * kf + kl) : 0;
            upto = (int)wave_incl_scan((uint32_t)mine);
            if (__builtin_amdgcn_readlane(upto, 63) <= TREE_WGS) break;
        }
        const unsigned long long here = __builtin_amdgcn_ballot_w64(wg >= upto - mine && wg < upto);
        if (here) {
            b = __ffsll(here) - 1;
            auto of = [&](int v) { return __builtin_amdgcn_readlane(v, b); };
            q = TreeSequence{of(own.t0), of(own.n), of(own.base), of(own.end)};
            kf = of(kf);
            kl = of(kl);
            const int qt = of(c.qt), tiles = of(c.tiles);
            uint32_t in = wg - of(upto - mine);
            const uint32_t head = (qt - 1) * kf + kl, in_head = in % head;
            tile = qt > 1 ? min((int)(in_head / (uint32_t)kf), qt - 1) : 0;
            in = (in - in_head) / head;  // (the KV head)
            const int part = (int)in_head - tile * kf, ns = tile == qt - 1 ? kl : kf;
            place(q, b, (int)in, tile, (int)((uint32_t)(tiles * part) / (uint32_t)ns), (int)((uint32_t)(tiles * (part + 1)) / (uint32_t)ns), tiles);
            if (part == 0 && ns > 1) split = TreeSplit{wg + ns - 1, w.members * G, w.first, w.h};
            again = true;
        }
        __syncthreads();
    } else {
        int64_t mine = a.Hkv * TreeCosts(own, G, units).head();
        for (int k = b0 + 1; k < b0 + per; ++k) mine += a.Hkv * TreeCosts(tree_sequence(a, k), G, units).head();
        if (few && wave > 0) mine = 0;
        int64_t upto = mine;
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t v = __shfl_up(upto, d, 64);
            if (lane >= d) upto += v;
        }
        if (lane == 63) s.pre[wave] = upto;
        __syncthreads();
        int64_t front = 0;
        for (int k = 0; k < wave; ++k) front += s.pre[k];
        __syncthreads();
        s.pre[tid + 1] = front + upto;
        if (tid == 0) s.pre[0] = 0;
        __syncthreads();
        total = s.pre[256];
        pieces = (int)max((int64_t)1, min((int64_t)TREE_WGS, total / LEAST));
        pos = p0 = quotient(total * min(wg, pieces), pieces);
        p1 = quotient(total * min(wg + 1, pieces), pieces);
        h = a.Hkv;
        again = pos < p1;
    }
    int seen_of = -1, seen_first = -1;
    while (again) {
        if (whole) {
            again = false;
        } else {
            if (h >= a.Hkv) {  // the sequence that has the unit at pos
                __syncthreads();
                if (s.pre[tid] <= pos && pos < s.pre[tid + 1]) {
                    int k = b0;
                    int64_t at = s.pre[tid];
                    TreeSequence mine = own;
                    for (int64_t c = a.Hkv * TreeCosts(mine, G, units).head(); at + c <= pos; c = a.Hkv * TreeCosts(mine, G, units).head()) {
                        at += c;
                        mine = tree_sequence(a, ++k);
                    }
                    s.at = at;
                    s.b = k;
                    s.q = mine;
                }
                __syncthreads();
                q = TreeSequence{__builtin_amdgcn_readfirstlane(s.q.t0), __builtin_amdgcn_readfirstlane(s.q.n),
                                 __builtin_amdgcn_readfirstlane(s.q.base), __builtin_amdgcn_readfirstlane(s.q.end)};
                b = __builtin_amdgcn_readfirstlane(s.b);
                const TreeCosts c(q, G, units);
                const int64_t head = c.head(), full = c.unit(c.full);
                h = __builtin_amdgcn_readfirstlane((int)quotient(pos - s.at, head));
                tile = __builtin_amdgcn_readfirstlane(min((int)quotient(pos - s.at - h * head, full), c.qt - 1));
                u0 = s.at + h * head + tile * full;
            }
            const TreeCosts c(q, G, units);
            const int weight = tile == c.qt - 1 ? c.last : c.full;
            const int64_t u1 = u0 + c.unit(weight);
            place(q, b, h, tile, p0 <= u0 ? 0 : c.tile_at(p0 - u0, weight), p1 >= u1 ? c.tiles : c.tile_at(p1 - u0, weight), c.tiles);
            pos = u0 = u1;
            if (++tile == c.qt) {
                tile = 0;
                ++h;
            }
            again = pos < p1;
            if (w.t1 == w.t0) continue;
            if (w.t0 == 0 && !w.final)  // (to the last workgroup whose piece begins below u1)
                split = TreeSplit{(int)quotient(u1 * pieces - 1, total), w.members * G, w.first, w.h};
        }
        if (w.end == 0) {  // no rows at all
            for (int i = tid; i < w.members * G * (HATA_D / 4); i += 256) {
                const int r = i / (HATA_D / 4);
                store_output(a.out, a.out_f32, (int64_t)(w.first * a.Hq + w.h * G + s.row[r]) * HATA_D + i % (HATA_D / 4) * 4,
                             make_float4(0.f, 0.f, 0.f, 0.f));
            }
            continue;
        }
        if (w.t1 * PREFIX_TILE > w.base && (seen_of != b || seen_first != w.first)) {  // (the same for all heads)
            tree_seen(a, w, s.seen);
            seen_of = b;
            seen_first = w.first;
        }
        __syncthreads();
        w.first = __builtin_amdgcn_readfirstlane(w.first);
        for (int* v : {&w.members, &w.t0, &w.t1, &w.h, &w.lead, &w.item, &w.base, &w.end}) *v = __builtin_amdgcn_readfirstlane(*v);
        const int rows = w.members * G;
        if (SMALL || rows <= 32) shared_rows<1, 1, true>(a, w, smem, tables);
        else if (rows <= 64) shared_rows<1, 2, true>(a, w, smem, tables);
        else if (rows <= 128) shared_rows<2, 2, true>(a, w, smem, tables);
        else shared_rows<4, 2, true>(a, w, smem, tables);
        __syncthreads();  // (the LDS is used anew)
    }
    if (tid == 0) a.splits[wg] = split;
}

// The results of the units that several workgroups have, joined: eight query rows a workgroup, half a wave each.  A launch of its own,
// because a workgroup that waited for the others' parts would need them resident.  Bound by latencies: 4 us of nothing but the
// launch, the record, the parts; 8.5 for 150 units of two parts (15 with 16 parts requested together, whatever there were, in 121
// registers, by which half as many workgroups were resident; 10.3 with half the workgroups and twice the rows each).
#define TREE_MERGE_ROWS 8
#define TREE_MERGE_BATCH 8  // partial results requested together
#define TREE_MERGE_FEW 4     // up to so many without LDS
// (A unit's groups take turns on the XCDs.  With those of unit i all on XCD i % 8, units of 32 parts, which begin in workgroups 0, 32,
// 64 .., are all on one: eight of them with 256 query rows 47 us instead of 9, 150 units of two parts 23 us instead of 15; each on the XCD that
// has its parts in its L2 11 and 22 us)
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeArgs a) {
    __shared__ float s_f[TREE_MERGE_ROWS][TREE_WGS];
    const int group = blockIdx.y, unit = (blockIdx.x - group) & (TREE_WGS - 1);
    const TreeSplit u = a.splits[unit];
    const int row = threadIdx.x >> 5, r = group * TREE_MERGE_ROWS + row, lane = threadIdx.x & 31;
    if (u.last < 0 || group * TREE_MERGE_ROWS >= u.rows) return;
    const int at = min(r, u.rows - 1), ns = u.last - unit + 1;
    const uint32_t size = a.part_rows * (HATA_D + 2);  // (all of them: below 2^25 floats)
    const float* part = a.part + 2 * (int64_t)unit * size;
    auto of_split = [&](int s) { return (s ? 2 * s : 1) * size; };
    auto weight = [](float x, float top) { return x == HATA_NEG_INF ? (top == HATA_NEG_INF ? 1.f : 0.f) : fast_exp2(x - (top == HATA_NEG_INF ? 0.f : top)); };
    auto sums_of = [&](int s) { return *reinterpret_cast<const float2*>(part + (of_split(s) + a.part_rows * HATA_D + 2 * at)); };
    float top = HATA_NEG_INF, l = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    // parts s0 .. s0 + N - 1: requested, and added (no branch: requests behind one would go out one by one.  32 partial results of 256 query
    // rows and eight heads 72 us that way)
    auto load = [&](auto& v, int s0) {
        int j = 0;
        for (float4& x : v) x = *reinterpret_cast<const float4*>(part + (of_split(min(s0 + j++, ns - 1)) + at * HATA_D + 4 * lane));
    };
    auto add = [&](const float4& v, float f, bool here) {
        const uint32_t there = here ? ~0u : 0u;
        auto one = [&](float& sum, float x) { sum = fmaf(f, __uint_as_float(__float_as_uint(x) & there), sum); };
        one(o.x, v.x); one(o.y, v.y); one(o.z, v.z); one(o.w, v.w);
    };
    if (ns <= TREE_MERGE_FEW) {
        float2 ml[TREE_MERGE_FEW];
        float4 v[TREE_MERGE_FEW];
#pragma unroll
        for (int s = 0; s < TREE_MERGE_FEW; ++s) ml[s] = sums_of(min(s, ns - 1));
        load(v, 0);
#pragma unroll
        for (int s = 0; s < TREE_MERGE_FEW; ++s) top = fmaxf(top, ml[s].x);
#pragma unroll
        for (int s = 0; s < TREE_MERGE_FEW; ++s) {
            const float f = weight(ml[s].x, top);
            l = s < ns ? fmaf(f, ml[s].y, l) : l;
            add(v[s], f, s < ns);
        }
    } else {
        float2 ml[TREE_WGS / 32];
#pragma unroll
        for (int j = 0; j < TREE_WGS / 32; ++j) {
            const int s = 32 * j + lane;
            ml[j] = make_float2(HATA_NEG_INF, 0.f);
            if (s < ns) ml[j] = sums_of(s);
            top = fmaxf(top, ml[j].x);
        }
        float4 v[TREE_MERGE_BATCH];
        load(v, 0);  // (on their way with the references)
        for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
#pragma unroll
        for (int j = 0; j < TREE_WGS / 32; ++j) {
            const int s = 32 * j + lane;
            const float f = weight(ml[j].x, top);
            if (s < ns) {
                s_f[row][s] = f;
                l = fmaf(f, ml[j].y, l);
            }
        }
        for (int m = 16; m; m >>= 1) l += __shfl_xor(l, m, 64);
        __syncthreads();
        for (int s0 = 0; s0 < ns; s0 += TREE_MERGE_BATCH) {
            if (s0) load(v, s0);
#pragma unroll
            for (int j = 0; j < TREE_MERGE_BATCH; ++j) add(v[j], s_f[row][min(s0 + j, ns - 1)], s0 + j < ns);
        }
    }
    if (r >= u.rows) return;
    const float f = 1.f / l;
    o = l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o.x * f, o.y * f, o.z * f, o.w * f);  // (NaN too)
    store_output(a.out, a.out_f32, ((int64_t)(u.first + r / a.G) * a.Hq + u.h * a.G + r % a.G) * HATA_D + 4 * lane, o);
}

// Query rows of a unit are never more than this
static int tree_part_rows(int G, int max_draft) { return (int64_t)max_draft * G <= 32 ? 32 : TREE_ROWS; }
// [a record a workgroup][two partial results a workgroup]
#define TREE_SPLITS_BYTES (TREE_WGS * sizeof(TreeSplit))
size_t tree_scratch_bytes(int G, int max_draft) {
    return TREE_SPLITS_BYTES + (size_t)2 * TREE_WGS * tree_part_rows(G, max_draft) * (HATA_D + 2) * 4;
}

hipError_t prepare_tree() {
    for (const void* fn : {(const void*)tree_kernel<true>, (const void*)tree_kernel<false>}) {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, PREFIX_LDS);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_tree(const TreeArgs& args, void* scratch, hipStream_t s) {
    TreeArgs a = args;
    a.part_rows = tree_part_rows(a.G, a.max_draft);
    a.splits = (TreeSplit*)scratch;
    a.part = (float*)((char*)scratch + TREE_SPLITS_BYTES);
    hipLaunchKernelGGL((a.part_rows == 32 ? tree_kernel<true> : tree_kernel<false>), dim3(TREE_WGS), dim3(256), PREFIX_LDS, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const int rows = std::min(a.max_draft * a.G, a.part_rows);
    hipLaunchKernelGGL(tree_merge_kernel, dim3(TREE_WGS, (rows + TREE_MERGE_ROWS - 1) / TREE_MERGE_ROWS), dim3(256), 0, s, a);
    return hipGetLastError();
}

// ---- the accepted path ----
//
// A workgroup has some KV heads of a sequence.  The rows' places are looked up once for all of them; then rows go as many at a time as the
// threads have registers for, all read before the first is written: a path's rows move to the front only, so rows that are still to be
// read are never written.  Bound by latency: lengths and path, places, rows, one after the other: 8 sequences 3.5 us (the host needs 5.5 a
// call), 256 sequences with paths of up to 12, eight KV heads,
// r = 256, 5.6 us (a workgroup a head, every place looked up by every thread, 19).
__global__ __launch_bounds__(256) void keep_rows_kernel(const KeepRows a) {
    __shared__ int s_from[HATA_TREE_MAX_DRAFT], s_to[HATA_TREE_MAX_DRAFT];  // row of the first KV head in the pools; -1: is there already
    __shared__ int s_kept;
    const int tid = threadIdx.x, b = blockIdx.y, h0 = blockIdx.x * a.heads, heads = min(a.heads, a.Hkv - h0);
    const int* path = a.path + (int64_t)b * a.max_path;
    const int j = tid < a.max_path ? path[tid] : -1, before = tid > 0 && tid < a.max_path ? path[tid - 1] : -1;
    const int L = clampi(a.seq_len[b], 0, a.L_cap), base = clampi(a.base[b], 0, L);
    const int most = clampi(a.n_path[b], 0, min(a.max_path, HATA_TREE_MAX_DRAFT));
    if (tid == 0) s_kept = most;
    __syncthreads();
    if (tid < most && (j < 0 || j >= L - base || before >= j)) atomicMin(&s_kept, tid);
    __syncthreads();
    const int kept = s_kept;
    if (tid < kept) {
        s_from[tid] = pool_row(a.pv, b, base + j, 0, a.Hkv);
        s_to[tid] = j == tid ? -1 : pool_row(a.pv, b, base + tid, 0, a.Hkv);
    }
    if (blockIdx.x == 0 && tid == 0) a.seq_len_out[b] = base + kept;
    __syncthreads();
    // A turn: 2048 pieces of 16 bytes, 16 of K and 16 of V a row and head, and 512 words of codes, eight a row and head (heads to a
    // power of two)
    const int hs = heads > 1 ? 32 - __clz(heads - 1) : 0, rows = max(64 >> hs, 1);
    for (int i0 = 0; i0 < kept; i0 += rows)
        for (int e0 = 0; e0 < 32 << hs; e0 += 2048) {  // (more than once with 128 heads and more: a part of the heads at a time)
            uint4 v[8];
            uint32_t code[2];
            uint16_t* at[8];
            uint32_t* code_at[2];
            auto place = [&](int e, int shift, int& i, int& h) {  // items of 1 << shift a row and head
                i = i0 + (e >> (shift + hs));
                h = h0 + (e >> shift & ((1 << hs) - 1));
                return i < min(kept, i0 + rows) && h < h0 + heads && s_to[i] >= 0;
            };
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int e = e0 + u * 256 + tid;
                int i, h;
                at[u] = nullptr;
                v[u] = make_uint4(0, 0, 0, 0);
                if (place(e, 5, i, h)) {
                    uint16_t* pool = (e & 16 ? a.V : a.K) + (e & 15) * 8;
                    v[u] = *reinterpret_cast<const uint4*>(pool + (s_from[i] + ((int64_t)h << a.pv.shift)) * HATA_D);
                    at[u] = pool + (s_to[i] + ((int64_t)h << a.pv.shift)) * HATA_D;
                }
            }
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int e = e0 / 4 + u * 256 + tid;
                int i, h;
                code_at[u] = nullptr;
                code[u] = 0;
                if (a.codes && (e & 7) < a.Wd && place(e, 3, i, h)) {
                    code[u] = a.codes[(s_from[i] + ((int64_t)h << a.pv.shift)) * a.Wd + (e & 7)];
                    code_at[u] = a.codes + (s_to[i] + ((int64_t)h << a.pv.shift)) * a.Wd + (e & 7);
                }
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (at[u]) *reinterpret_cast<uint4*>(at[u]) = v[u];
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (code_at[u]) *code_at[u] = code[u];
        }
}

hipError_t launch_keep_rows(const KeepRows& args, int B, hipStream_t s) {
    KeepRows a = args;
    a.heads = 1;  // of a workgroup: two rounds of them at most
    while ((int64_t)B * ((a.Hkv + a.heads - 1) / a.heads) > 512 && a.heads < a.Hkv) a.heads *= 2;
    hipLaunchKernelGGL(keep_rows_kernel, dim3((a.Hkv + a.heads - 1) / a.heads, B), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace hata
