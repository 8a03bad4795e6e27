// Attention of drafted tokens on block tables (hata_dense_tree_paged), and the rows of the accepted ones (hata_keep_rows).
#include <algorithm>
#include "hata_attn_core.h"
#include "hata_device.h"
#include "hata_internal.h"
#include "hata_shared_rows.h"

namespace hata {

// Row n of sequence b in the pools: the row of head h of its page is row_of(n) * 1 (in rows of HATA_D values)
__device__ __forceinline__ int pool_row(const PageView& pv, int b, int n, int h, int Hkv) {
    const int page = clampi(pv.table[(int64_t)b * pv.max_blocks + (n >> pv.shift)], 0, pv.n_pages - 1);
    return ((page * Hkv + h) << pv.shift) + (n & ((1 << pv.shift) - 1));
}

// ---- which workgroup does what ----
//
// A unit is a KV head of a tile of a sequence's tokens (M / G of them: M query rows).  Every workgroup works out for itself the shortest
// run of rows (in tiles of PREFIX_TILE) at which the launch's workgroups suffice, one per (unit, run); the tiles of tokens of a run are
// neighbours on one XCD.  Batches of more than TREE_SPLIT_B sequences have enough units: a run each.
#define TREE_SPLIT_B 4096
struct TreeRun { int members, tiles, split, ns, h, first, lead, item, base, end, draft0, n; };
struct TreeSequence { int t0, n, base, end, tiles, qt; };

__device__ __forceinline__ TreeSequence tree_sequence(const TreeArgs& a, int mpt, int b) {
    TreeSequence q = {0, 0, 0, 0, 0, 0};
    if (b >= a.B) return q;
    q.t0 = clampi(a.token_start[b], 0, a.n_tokens);
    q.n = clampi(clampi(a.token_start[b + 1], 0, a.n_tokens) - q.t0, 0, a.max_draft);
    const int L = clampi(a.seq_len[b], 0, a.L_cap);
    q.base = clampi(a.base[b], 0, L);
    q.end = min(L, q.base + q.n);
    q.tiles = max(1, (q.end + PREFIX_TILE - 1) / PREFIX_TILE);
    q.qt = (q.n + mpt - 1) / mpt;
    return q;
}

// smem: [min(B, TREE_SPLIT_B)] words
__device__ __forceinline__ bool tree_share(const TreeArgs& a, int mpt, uint32_t* lds, TreeRun& w) {
    const int tid = threadIdx.x, lane = tid & 63, item = (int)((blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8);
    const bool split = a.B <= TREE_SPLIT_B;
    if (split) {
        for (int b = tid; b < a.B; b += 256) {
            const TreeSequence q = tree_sequence(a, mpt, b);
            lds[b] = (uint32_t)q.tiles | (uint32_t)q.qt << 20;
        }
        __syncthreads();
    }
    int run = 0x3fffffff;
    auto packed = [&](int b) {
        if (split) return b < a.B ? lds[b] : 0u;
        const TreeSequence q = tree_sequence(a, mpt, b);
        return (uint32_t)q.tiles | (uint32_t)q.qt << 20;
    };
    auto splits = [&](uint32_t p) { return min((int)((p & 0xfffffu) + run - 1) / run, PREFIX_MAX_SPLITS); };
    float units = 0.f;
    if (split) {
        float all = 0.f, longest = 0.f;
        for (int b = lane; b < a.B; b += 64) {
            const uint32_t p = lds[b];
            units += (float)(p >> 20);
            all += (float)(p >> 20) * (float)(p & 0xfffffu);
            if (p >> 20) longest = fmaxf(longest, (float)(p & 0xfffffu));
        }
        all = wave_sum64(all);
        longest = wave_max64(longest);
        for (run = max(1, (int)ceilf(all * (float)a.Hkv / (float)gridDim.x)); run < (int)longest; run += max(1, run >> 4)) {
            float items = 0.f;  // (below 2^24)
            for (int b = lane; b < a.B; b += 64) {
                const uint32_t p = lds[b];
                items += (float)((p >> 20) * splits(p));
            }
            if (wave_sum64(items) * (float)a.Hkv <= (float)gridDim.x) break;
        }
    } else if (blockIdx.x == 0) {
        for (int b0 = 0; b0 < a.B; b0 += 64) units += (float)(packed(b0 + lane) >> 20);
    }
    if (blockIdx.x == 0) {
        units = wave_sum64(units);
        if (tid == 0) *a.n_units = (int)units * a.Hkv;
    }
    int base = 0, unit = 0;
    bool found = false;
    for (int b0 = 0; b0 < a.B && !found; b0 += 64) {
        const uint32_t p = packed(b0 + lane);
        const int qt = (int)(p >> 20), ns = splits(p), mine = a.Hkv * qt * ns;
        const int upto = base + (int)wave_incl_scan((uint32_t)mine), at = upto - mine;
        const int unit_upto = unit + (int)wave_incl_scan((uint32_t)(a.Hkv * qt));
        const unsigned long long here = __builtin_amdgcn_ballot_w64(item >= at && item < upto);
        if (here) {
            found = true;
            const int l = __ffsll(here) - 1, b = b0 + l;
            const int in = item - __builtin_amdgcn_readlane(at, l), qts = __builtin_amdgcn_readlane(qt, l), u0 = __builtin_amdgcn_readlane(unit_upto - a.Hkv * qt, l);
            w.ns = __builtin_amdgcn_readlane(ns, l);
            const int q = in % qts;
            w.split = in / qts % w.ns;
            w.h = in / (qts * w.ns);
            const TreeSequence s = tree_sequence(a, mpt, b);
            w.tiles = s.tiles;
            w.lead = b;
            w.item = item;
            w.base = s.base;
            w.end = s.end;
            w.n = s.n;
            w.draft0 = q * mpt;
            w.first = s.t0 + w.draft0;
            w.members = min(mpt, s.n - w.draft0);
            const int u = u0 + w.h * qts + q;
            if (w.split == 0 && tid == 0 && u < a.max_units) a.units[u] = TreeUnit{item, qts, w.ns, w.members * a.G, w.first, w.h};
        }
        base = __builtin_amdgcn_readlane(upto, 63);
        unit = __builtin_amdgcn_readlane(unit_upto, 63);
    }
    __syncthreads();  // (the LDS is used anew)
    return found;
}

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

template <int WQ, int T>
__global__ __launch_bounds__(256, 1) void tree_kernel(const TreeArgs a) {
    constexpr int M = 32 * T * WQ;
    extern __shared__ __attribute__((aligned(16))) char smem[];
    __shared__ uint32_t s_seen[M * SEEN_WORDS];
    TreeRun w;
    if (!tree_share(a, M / a.G, reinterpret_cast<uint32_t*>(smem), w)) return;
    if (w.end == 0) {  // no rows at all
        const int G = a.G;
        for (int i = threadIdx.x; i < w.members * G * (HATA_D / 4); i += 256) {
            const int r = i / (HATA_D / 4);
            store_output(a.out, a.out_f32, ((int64_t)(w.first + r / G) * a.Hq + w.h * G + r % G) * HATA_D + i % (HATA_D / 4) * 4,
                         make_float4(0.f, 0.f, 0.f, 0.f));
        }
        return;
    }
    if ((int64_t)w.tiles * (w.split + 1) / w.ns * PREFIX_TILE > w.base) tree_seen(a, w, s_seen);
    __syncthreads();
    shared_rows<WQ, T, true>(a, w, smem, s_seen);
}

// The runs' results joined: eight query rows a workgroup, half a wave each
#define TREE_MERGE_ROWS 8
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeArgs a, int M) {
    __shared__ float s_f[TREE_MERGE_ROWS][PREFIX_MAX_SPLITS];
    if ((int)blockIdx.x >= *a.n_units) return;
    const TreeUnit u = a.units[blockIdx.x];
    const int row = threadIdx.x >> 5, r = blockIdx.y * TREE_MERGE_ROWS + row, lane = threadIdx.x & 31;
    if (u.ns == 1 || (int)blockIdx.y * TREE_MERGE_ROWS >= u.rows) return;
    const int at = min(r, u.rows - 1);
    const int64_t size = (int64_t)M * (HATA_D + 2), step = u.step * size;
    const float* part = a.part + u.item * size;
    float top = HATA_NEG_INF, l = 0.f;
    float2 ml[PREFIX_MAX_SPLITS / 32];
#pragma unroll
    for (int j = 0; j < PREFIX_MAX_SPLITS / 32; ++j) {
        const int s = 32 * j + lane;
        ml[j] = make_float2(HATA_NEG_INF, 0.f);
        if (s < u.ns) ml[j] = *reinterpret_cast<const float2*>(part + s * step + M * HATA_D + 2 * at);
        top = fmaxf(top, ml[j].x);
    }
    for (int m = 16; m; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
    const float sub = top == HATA_NEG_INF ? 0.f : top;
#pragma unroll
    for (int j = 0; j < PREFIX_MAX_SPLITS / 32; ++j) {
        const int s = 32 * j + lane;
        const float f = ml[j].x == HATA_NEG_INF ? (top == HATA_NEG_INF ? 1.f : 0.f) : fast_exp2(ml[j].x - sub);
        if (s < u.ns) {
            s_f[row][s] = f;
            l = fmaf(f, ml[j].y, l);
        }
    }
    for (int m = 16; m; m >>= 1) l += __shfl_xor(l, m, 64);
    __syncthreads();
    const float* p = part + at * HATA_D + 4 * lane;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = 0; s0 < u.ns; s0 += 8) {
        float4 v[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = *reinterpret_cast<const float4*>(p + min(s0 + j, u.ns - 1) * step);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (s0 + j >= u.ns) break;
            const float f = s_f[row][s0 + j];
            o.x = fmaf(f, v[j].x, o.x); o.y = fmaf(f, v[j].y, o.y); o.z = fmaf(f, v[j].z, o.z); o.w = fmaf(f, v[j].w, o.w);
        }
    }
    if (r >= u.rows) return;
    const float f = l == 0.f ? 0.f : 1.f / l;
    o.x *= f; o.y *= f; o.z *= f; o.w *= f;
    store_output(a.out, a.out_f32, ((int64_t)(u.first + r / a.G) * a.Hq + u.h * a.G + r % a.G) * HATA_D + 4 * lane, o);
}

// Query rows of a workgroup, from the mean of the sequences (what the host knows)
static int tree_rows(int B, int G, int n_tokens) {
    const int64_t rows = ((int64_t)n_tokens * G + B - 1) / B;
    return rows <= 32 ? 32 : rows <= 64 ? 64 : rows <= 448 ? 128 : 256;
}
static int64_t tree_units(int B, int Hkv, int G, int n_tokens, int M) {
    const int mpt = M / G;
    return (n_tokens + (int64_t)B * (mpt - 1)) / mpt * Hkv;
}
static int64_t tree_wgs(int64_t units) { return std::max((int64_t)256, (units + 255) / 256 * 256); }

// [the number of units][their records][partial results], for any tile of query rows that fewer tokens or sequences may go by
static size_t tree_part_offset(int64_t units) { return 256 + ((size_t)units * sizeof(TreeUnit) + 255) / 256 * 256; }
size_t tree_scratch_bytes(int B, int Hkv, int G, int n_tokens, int) {
    size_t most = 0;
    for (int M : {32, 64, 128, 256}) {
        const int64_t units = tree_units(B, Hkv, G, n_tokens, M);
        most = std::max(most, tree_part_offset(units) + (size_t)tree_wgs(units) * M * (HATA_D + 2) * 4);
    }
    return most;
}

hipError_t prepare_tree() {
    for (const void* fn : {(const void*)tree_kernel<1, 1>, (const void*)tree_kernel<1, 2>, (const void*)tree_kernel<2, 2>, (const void*)tree_kernel<4, 2>}) {
        const hipError_t e = hipFuncSetAttribute(fn, hipFuncAttributeMaxDynamicSharedMemorySize, PREFIX_LDS);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t launch_tree(const TreeArgs& args, void* scratch, hipStream_t s) {
    TreeArgs a = args;
    const int M = tree_rows(a.B, a.G, a.n_tokens);
    const int64_t units = tree_units(a.B, a.Hkv, a.G, a.n_tokens, M);
    a.n_units = (int*)scratch;
    a.units = (TreeUnit*)((char*)scratch + 256);
    a.part = (float*)((char*)scratch + tree_part_offset(units));
    a.max_units = (int)units;
    const dim3 grid((unsigned)tree_wgs(units));
    hipLaunchKernelGGL((M == 32 ? tree_kernel<1, 1> : M == 64 ? tree_kernel<1, 2> : M == 128 ? tree_kernel<2, 2> : tree_kernel<4, 2>), grid, dim3(256),
                       PREFIX_LDS, s, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || units == 0) return e;
    hipLaunchKernelGGL(tree_merge_kernel, dim3((unsigned)units, M / TREE_MERGE_ROWS), dim3(256), 0, s, a, M);
    return hipGetLastError();
}

// ---- the accepted path ----
//
// A workgroup has a KV head of a sequence.  Rows go KEEP_ROWS at a time, all read before the first is written: a path's rows move
// to the front only, so rows that are still to be read are never written.
#define KEEP_ROWS 32
__global__ __launch_bounds__(256) void keep_rows_kernel(const KeepRows a) {
    __shared__ int s_path[HATA_TREE_MAX_DRAFT], s_kept;
    const int tid = threadIdx.x, h = blockIdx.x, b = blockIdx.y;
    const int L = clampi(a.seq_len[b], 0, a.L_cap), base = clampi(a.base[b], 0, L);
    const int most = clampi(a.n_path[b], 0, min(a.max_path, HATA_TREE_MAX_DRAFT));
    if (tid == 0) s_kept = most;
    __syncthreads();
    const int* path = a.path + (int64_t)b * a.max_path;
    for (int i = tid; i < most; i += 256) {
        const int j = path[i];
        s_path[i] = j;
        if (j < 0 || j >= L - base || (i > 0 && path[i - 1] >= j)) atomicMin(&s_kept, i);
    }
    __syncthreads();
    const int kept = s_kept, col = tid & 31, r8 = tid >> 5;
    for (int i0 = 0; i0 < kept; i0 += KEEP_ROWS) {
        uint4 v[4];
        uint32_t code = 0;
        uint16_t* pool = (col < 16 ? a.K : a.V) + (col & 15) * 8;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + 8 * u + r8;
            if (i < kept) v[u] = *reinterpret_cast<const uint4*>(pool + (int64_t)pool_row(a.pv, b, base + s_path[i], h, a.Hkv) * HATA_D);
        }
        const int ic = i0 + (tid >> 3), w = tid & 7;
        const bool has_code = a.codes && ic < kept && w < a.Wd;
        if (has_code) code = a.codes[(int64_t)pool_row(a.pv, b, base + s_path[ic], h, a.Hkv) * a.Wd + w];
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int i = i0 + 8 * u + r8;
            if (i < kept && s_path[i] != i) *reinterpret_cast<uint4*>(pool + (int64_t)pool_row(a.pv, b, base + i, h, a.Hkv) * HATA_D) = v[u];
        }
        if (has_code && s_path[ic] != ic) a.codes[(int64_t)pool_row(a.pv, b, base + ic, h, a.Hkv) * a.Wd + w] = code;
        __syncthreads();
    }
    if (h == 0 && tid == 0) a.seq_len_out[b] = base + kept;
}

hipError_t launch_keep_rows(const KeepRows& a, int B, hipStream_t s) {
    hipLaunchKernelGGL(keep_rows_kernel, dim3(a.Hkv, B), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace hata
