// Decode attention over rows that a group of sequences has in common (Eq. 1 of the paper, block tables): read once for all of
// them.  For the query rows i of a group's members (member by member, the G heads of a KV head side by side) and a run of the
// common rows,
//   m_i = max_n s_in,  l_i = sum_n 2^(s_in - m_i),  o_i = sum_n 2^(s_in - m_i) V_n,   s_in = scale log2(e) q_i . K_n,
// which dense_kernel joins with the sequences' own rows.
//
//   - A workgroup of four waves has a tile of 64 WQ query rows and a run of rows.  A wave holds 64 query rows (operands and sums:
//     192 registers) and goes over 32 rows at a time on v_mfma_f32_32x32x16_bf16: S^T = K Q^T, O^T += V^T P^T.  In S^T a lane has 16
//     rows of ONE query row, which are what the second product wants from it as P: nothing crosses lanes.
//   - WQ waves share what they read (rows come into LDS by direct loads, 64 of K and of V a stage), 4 / WQ go over different rows.
//   - The maximum is followed loosely: a wave scales its sums only where a score passes the one in use by 2^8.
//   - Weights are rounded to bf16 (to nearest: half a step, 2^-8 relative; their sum is of the rounded ones), which halves the second
//     product against two terms, and the matrix cores are what bounds groups of more than some 200 query rows a KV head.
#include <algorithm>
#include "hata_attn_core.h"
#include "hata_device.h"
#include "hata_internal.h"

namespace hata {

typedef __attribute__((ext_vector_type(16))) float f32x16_t;
typedef __attribute__((ext_vector_type(2))) float f32x2_t;

#define PREFIX_TILE 64       // rows that runs are cut by; what is left of the common rows is read by every sequence itself
#define PREFIX_MAX_SPLITS 256
#define PREFIX_LDS (4 * 64 * (HATA_D + 4) * 4)  // the waves' sums at the end; before, the ring of stages

struct PrefixArgs {
    const uint16_t *q, *K, *V;
    const int32_t *seq_len, *group_start, *shared_len;
    int4* info;
    float* part;
    PageView pv;
    int B, Hq, Hkv, G, L_cap, n_groups;
    float scale_log2;
};

// ---- which workgroup does what ----
//
// Every workgroup works it out for itself: the groups' members, the rows they have in common, and the shortest run (in tiles) at
// which the launch's workgroups suffice, one per (group, KV head, tile of query rows, run).  The tiles of query rows of a run are
// neighbours on one XCD, whose L2 then serves all but the first of them.
struct PrefixShare { int g, h, split, ns, qt, tiles, item, first, members, lead; };

__device__ __forceinline__ bool prefix_share(const PrefixArgs& a, int mpt, int* lds, PrefixShare& w) {
    const int n = a.n_groups, tid = threadIdx.x, lane = tid & 63;
    int* start = lds;            // [n + 1] first member
    int* least = start + n + 1;  // [n] rows of the shortest member that has rows; afterwards tiles in common
    int* count = least + n;      // [n] members that have rows
    int* lead = count + n;       // [n] the first of them
    for (int i = tid; i <= n; i += 256) {
        start[i] = clampi(a.group_start[i], 0, a.B);
        if (i < n) { least[i] = 0x7fffffff; count[i] = 0; lead[i] = 0x7fffffff; }
    }
    __syncthreads();
    for (int o = 1; o <= n; o <<= 1) {  // ascending, whatever the caller gave
        int v[HATA_PREFIX_GROUPS / 256 + 1];
#pragma unroll
        for (int k = 0; k < HATA_PREFIX_GROUPS / 256 + 1; ++k) {
            const int i = tid + 256 * k;
            v[k] = i <= n ? max(start[i], i >= o ? start[i - o] : 0) : 0;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < HATA_PREFIX_GROUPS / 256 + 1; ++k)
            if (tid + 256 * k <= n) start[tid + 256 * k] = v[k];
        __syncthreads();
    }
    auto group_of = [&](int b) {  // -1: none
        if (b < start[0] || b >= start[n]) return -1;
        int lo = 0, c = n;  // the last group that begins at b or before
        while (c > 1) {
            const int half = c / 2;
            if (start[lo + half] <= b) { lo += half; c -= half; }
            else c = half;
        }
        return lo;
    };
    for (int b = start[0] + tid; b < start[n]; b += 256) {
        const int L = clampi(a.seq_len[b], 0, a.L_cap), g = group_of(b);
        if (L > 0) {
            atomicMin(&least[g], L);
            atomicAdd(&count[g], 1);
            atomicMin(&lead[g], b);
        }
    }
    __syncthreads();
    for (int g = tid; g < n; g += 256) least[g] = count[g] >= 2 ? max(min(a.shared_len[g], least[g]), 0) / PREFIX_TILE : 0;
    __syncthreads();
    auto qtiles = [&](int g) { return (start[g + 1] - start[g] + mpt - 1) / mpt; };
    auto splits = [&](int g, int run) { return min((least[g] + run - 1) / run, PREFIX_MAX_SPLITS); };
    int64_t all = 0;
    int longest = 1;
    for (int g0 = 0; g0 < n; g0 += 64) {
        const int g = g0 + lane;
        all += (int64_t)wave_sum64(g < n ? (float)qtiles(g) * least[g] : 0.f);
        longest = max(longest, (int)wave_max64(g < n ? (float)least[g] : 0.f));
    }
    const int wgs = gridDim.x;
    int run = (int)max((int64_t)1, (all * a.Hkv + wgs - 1) / wgs);
    for (;; run += max(1, run >> 3)) {
        uint32_t items = 0;
        for (int g0 = 0; g0 < n; g0 += 64) {
            const int g = g0 + lane;
            items += (uint32_t)__builtin_amdgcn_readlane((int)wave_incl_scan(g < n ? (uint32_t)(qtiles(g) * splits(g, run)) : 0u), 63);
        }
        if (items * (uint32_t)a.Hkv <= (uint32_t)wgs || run >= longest) break;
    }
    // this workgroup's item, and for the first workgroup where every sequence finds its group's partial results
    const int item = (int)((blockIdx.x % 8) * (gridDim.x / 8) + blockIdx.x / 8);
    int base = 0;
    w.g = -1;
    for (int g = 0; g < n; ++g) {
        const int qt = qtiles(g), ns = splits(g, run), items = a.Hkv * qt * ns;
        if (blockIdx.x == 0) {
            for (int b = start[g] + tid; b < start[g + 1]; b += 256) {
                const int i = b - start[g];
                const bool some = ns > 0 && clampi(a.seq_len[b], 0, a.L_cap) > 0;
                a.info[b] = some ? make_int4(least[g] * PREFIX_TILE, base + i / mpt, ns | (i % mpt * a.G) << 16, qt) : make_int4(0, 0, 0, 0);
            }
        }
        if (item >= base && item < base + items) {
            const int in = item - base;
            w.g = g; w.ns = ns; w.tiles = least[g]; w.item = item;
            w.qt = in % qt;
            w.split = in / qt % ns;
            w.h = in / (qt * ns);
            w.first = start[g] + w.qt * mpt;
            w.members = min(mpt, start[g + 1] - w.first);
            w.lead = lead[g];
        }
        base += items;
    }
    if (blockIdx.x == 0)
        for (int b = tid; b < a.B; b += 256)
            if (b < start[0] || b >= start[n]) a.info[b] = make_int4(0, 0, 0, 0);
    __syncthreads();  // (the LDS is used anew)
    // (in scalar registers from here on)
    for (int* v : {&w.g, &w.h, &w.split, &w.ns, &w.qt, &w.tiles, &w.item, &w.first, &w.members, &w.lead}) *v = __builtin_amdgcn_readfirstlane(*v);
    return w.g >= 0;
}

// 16-byte piece c of row r of a stage is at slot c ^ prefix_swizzle(r): 16 rows of one piece, and four rows of four pieces, are in
// 16 different slots, so that neither product's reads have bank conflicts
__device__ __forceinline__ int prefix_swizzle(int r) { return (r & 3) << 2 | (r >> 2 & 3); }

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
    auto request = [&](int s) {
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) {
            const int row = first_row(s, j), page = clampi(pages[j], 0, a.pv.n_pages - 1);
            const int64_t at = ((((int64_t)page * a.Hkv + w.h) << a.pv.shift) + (row & ((1 << a.pv.shift) - 1))) * HATA_D;
            const uint32_t dst = ring + (uint32_t)((s % NBUF) * STAGE * 512 + (wk * PART + (wq * BLOCKS + j) * 16) * 256);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                // (written as instructions: behind the compiler's builtin for it, every LDS read waits for all requests)
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst + i * 1024), "v"(off[i]), "s"(a.K + at) : "memory", "m0");
                asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst + STAGE * 256 + i * 1024), "v"(off[i]), "s"(a.V + at) : "memory", "m0");
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
    // the maxima in use, where these scores pass one by 2^8
    auto follow = [&](const f32x16_t (&sc)[2]) {
        float top[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            top[t] = sc[t][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top[t] = fmaxf(top[t], sc[t][i]);
            top[t] *= scale;
        }
        if (__builtin_amdgcn_ballot_w64(top[0] > m[0] + 8.f || top[1] > m[1] + 8.f) != 0ull) {
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                float x, y;
                swap32(top[t], x, y);
                const float to = fmaxf(fmaxf(x, y), m[t]);  // of both halves' rows
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
    auto weights = [&](const f32x16_t (&sc)[2], uint32_t (&p)[2][8]) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                f32x2_t e;
                e[0] = fast_exp2(fmaf(sc[t][2 * i], scale, -sub[t]));
                e[1] = fast_exp2(fmaf(sc[t][2 * i + 1], scale, -sub[t]));
                p[t][i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(e, bf16x2_t));
                l[t] = dot2_bf16(p[t][i], 0x3f803f80u, l[t]);
            }
    };
    auto values = [&](const char* vt, const uint32_t (&p)[2][8]) {
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
                for (int t = 0; t < 2; ++t)
                    acc[t][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                        vf, __builtin_bit_cast(bf16x8_t, make_uint4(p[t][4 * x], p[t][4 * x + 1], p[t][4 * x + 2], p[t][4 * x + 3])), acc[t][c], 0, 0, 0);
            }
    };
    auto at_stage = [&](int s) { return (const char*)smem + (s % NBUF) * STAGE * 512 + wk * PART * 256; };  // K; V is STAGE * 256 bytes behind

    for (int s = 0; s < NBUF - (WQ > 1); ++s)
        if (s < stages) request(s);
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int s = 0; s < 8; ++s)  // (used here, so that the wait for these loads is not in the loop)
            asm volatile("" : "+a"(qb[t][s].x), "+a"(qb[t][s].y), "+a"(qb[t][s].z), "+a"(qb[t][s].w));
    pin();
    if constexpr (WQ == 1) {
        // rows of this wave alone: nothing is waited for but its own requests
        for (int s = 0; s < stages; ++s) {
            if (s + 1 < stages) prefix_wait<BLOCKS * 8>();
            else prefix_wait<0>();
            if (k0 + s * STAGE + wk * PART < k1) {
                f32x16_t sc[2];
                uint32_t p[2][8];
                products(at_stage(s), sc);
                follow(sc);
                weights(sc, p);
                values(at_stage(s) + STAGE * 256, p);
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // every read of this stage has returned
            if (s + NBUF < stages) request(s + NBUF);
            pin();
        }
    } else {
        // The products of the next 32 rows stand beside the weights of these: matrix cores and vector ALU at work together
        f32x16_t sc[2], next[2];
        if (stages >= NBUF - 1) prefix_wait<(NBUF - 2) * BLOCKS * 8>();  // (so many were requested)
        else prefix_wait<0>();
        __syncthreads();
        products(at_stage(0), sc);
        for (int s = 0; s < stages; ++s) {
#pragma unroll
            for (int i = 0; i < SUBS; ++i) {
                uint32_t p[2][8];
                follow(sc);
                if (i + 1 < SUBS) {
                    products(at_stage(s) + (i + 1) * 32 * 256, next);
                } else if (s + 1 < stages) {
                    // stage s + 1 is there once only the one behind it is outstanding; everybody is done with stage s - 1
                    if (s + 2 < stages) prefix_wait<(NBUF - 3) * BLOCKS * 8>();
                    else prefix_wait<0>();
                    __syncthreads();
                    if (s + NBUF - 1 < stages) request(s + NBUF - 1);
                    products(at_stage(s + 1), next);
                }
                weights(sc, p);
                values(at_stage(s) + STAGE * 256 + i * 32 * 256, p);
#pragma unroll
                for (int t = 0; t < 2; ++t) sc[t] = next[t];
                pin();
            }
        }
    }

    // ---- the waves' sums, joined where they have the same query rows ----
    __syncthreads();  // the ring is no longer read
    float* s_acc = reinterpret_cast<float*>(smem);  // [wave][64][HATA_D + 4]
    __shared__ float s_m[4][64], s_l[4][64];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        float x, y;
        swap32(l[t], x, y);
        if (half == 0) { s_m[wave][32 * t + n] = m[t]; s_l[wave][32 * t + n] = x + y; }
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)  // acc[t][c][4 i + j]: channel 32 c + 8 i + 4 half + j of query row 32 t + n
                *reinterpret_cast<float4*>(&s_acc[(wave * 64 + 32 * t + n) * (HATA_D + 4) + 32 * c + 8 * i + 4 * half]) =
                    make_float4(acc[t][c][4 * i], acc[t][c][4 * i + 1], acc[t][c][4 * i + 2], acc[t][c][4 * i + 3]);
    }
    __syncthreads();
    float* out = a.part + (int64_t)w.item * (M * (HATA_D + 2));
    for (int i = tid; i < rows * (HATA_D / 4); i += 256) {
        const int r = i / (HATA_D / 4), c4 = i % (HATA_D / 4) * 4, w0 = r / 64, r0 = r % 64;
        float top = s_m[w0][r0], sum = 0.f;
#pragma unroll
        for (int k = 1; k < WK; ++k) top = fmaxf(top, s_m[w0 + k * WQ][r0]);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < WK; ++k) {
            const int wv = w0 + k * WQ;
            const float f = s_m[wv][r0] == HATA_NEG_INF ? 0.f : fast_exp2(s_m[wv][r0] - top);
            const float4 v = *reinterpret_cast<const float4*>(&s_acc[(wv * 64 + r0) * (HATA_D + 4) + c4]);
            // (a wave whose scores were all -inf may hold NaN there, of infinite values; it counts if no other score does)
            if (f != 0.f || top == HATA_NEG_INF) {
                const float g = top == HATA_NEG_INF ? 1.f : f;
                o.x = fmaf(g, v.x, o.x); o.y = fmaf(g, v.y, o.y); o.z = fmaf(g, v.z, o.z); o.w = fmaf(g, v.w, o.w);
                sum = fmaf(g, s_l[wv][r0], sum);
            }
        }
        *reinterpret_cast<float4*>(out + r * HATA_D + c4) = o;
        if (c4 == 0) *reinterpret_cast<float2*>(out + M * HATA_D + 2 * r) = make_float2(top, sum);
    }
}

// Query rows of a workgroup (waves with rows of their own): from the mean of the groups, 64, 128 or 256
static int prefix_waves(int64_t rows_per_group) { return rows_per_group <= 64 ? 1 : rows_per_group <= 128 ? 2 : 4; }

// Workgroups of a launch: one per compute unit, or as many as the (tile of query rows, KV head) need
static int64_t prefix_wgs(int B, int Hkv, int G, int n_groups, int waves) {
    const int mpt = 64 * waves / G;
    const int64_t tiles = (B + (int64_t)n_groups * (mpt - 1)) / mpt * Hkv;
    return std::max((int64_t)256, (tiles + 255) / 256 * 256);
}

size_t prefix_part_floats(int B, int Hkv, int G) {
    if (B < 2) return 0;
    size_t most = 0;
    for (int waves = 1; waves <= 4; waves *= 2) {
        // the most groups that go by so many waves
        const int64_t groups = waves == 1 ? std::min(B, HATA_PREFIX_GROUPS) : std::min((int64_t)std::min(B, HATA_PREFIX_GROUPS), (int64_t)B * G / (32 * waves));
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
    a.info = (int4*)c->prefix_info;
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
