// Decode attention of many query rows over rows that they have in common (hata_prefix.hip: of sequences behind one prompt,
// hata_tree.hip: of one sequence's drafted tokens): sums l_i and o_i of the weights 2^(s_in - m_i) of a run of rows n.
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
#pragma once
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

__device__ __forceinline__ void store_output(uint16_t* out, float* out_f32, int64_t at, float4 o) {
    f32x2_t lo, hi;
    lo[0] = o.x; lo[1] = o.y; hi[0] = o.z; hi[1] = o.w;
    *reinterpret_cast<uint2*>(out + at) = make_uint2(__builtin_bit_cast(uint32_t, __builtin_convertvector(lo, bf16x2_t)),
                                                     __builtin_bit_cast(uint32_t, __builtin_convertvector(hi, bf16x2_t)));
    if (out_f32) *reinterpret_cast<float4*>(out_f32 + at) = o;
}

// What a workgroup of four waves has to do: the query rows of w.members sequences or tokens (packed rows w.first .. of q) and KV head w.h, and
// of the rows of sequence w.lead's table split w.split of w.ns of w.tiles tiles; smem: PREFIX_LDS bytes.  The sums go to partial result
// w.item, [M][HATA_D], then [M][2] (reference, sum).
// WQ: waves with query rows of their own, T: of 32 query rows of a wave, one or two.  A stage is 4 / WQ parts (one per wave with the same
// query rows) of PART rows, K and V.
// DRAFT: tiles w.t0 .. w.t1 - 1 of w.end rows, the last ones of which, from w.base on, are seen by those members only whose bit is set in `seen`
// [members][SEEN_WORDS] (LDS; no bit of a row from w.end on is); w.final: no other workgroup has rows of these query rows, the results go to
// a.out.  Partial results are a.part_rows high.
#define SEEN_WORDS 9  // of 256 drafted rows; the last is 0
struct DraftTables {   // in LDS
    const uint32_t* seen;
    const int *row, *member;  // of query row r: r / G * Hq + r % G, r / G
};
template <int WQ, int T, bool DRAFT, class Args, class Work>
__device__ __forceinline__ void shared_rows(const Args& a, const Work& w, char* smem, const DraftTables& tables = {}) {
    static_assert(T == 2 || WQ == 1, "waves with 32 query rows have the same ones");
    constexpr int WK = 4 / WQ, PART = WQ == 4 ? 64 : 32, STAGE = WK * PART, SUBS = PART / 32;
    constexpr int NBUF = 256 / STAGE;                                // stages in LDS: 128 KB
    constexpr int BLOCKS = PART / WQ / 16;                           // blocks of 16 rows a wave requests of a stage, K and V
    constexpr int M = 32 * T * WQ;
    int tid = threadIdx.x;
    if constexpr (DRAFT) asm volatile("" : "+v"(tid));  // (nothing is kept from one call of a kernel's loop to the next)
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wq = wave % WQ, wk = wave / WQ, n = lane & 31, half = lane >> 5;
    const int G = a.G, rows = w.members * G;
    // rows of this workgroup, in tiles of 64; of a stage of 128 that reaches over the end the waves behind it have nothing to do
    int t0, t1, k1;
    [[maybe_unused]] int base = 0, end = 0;
    if constexpr (DRAFT) {
        t0 = w.t0;
        t1 = w.t1;
        base = w.base;
        end = w.end;
        k1 = min(t1 * PREFIX_TILE, end);
    } else {
        t0 = (int)((int64_t)w.tiles * w.split / w.ns);
        t1 = (int)((int64_t)w.tiles * (w.split + 1) / w.ns);
        k1 = t1 * PREFIX_TILE;
    }
    const int k0 = t0 * PREFIX_TILE, stages = (k1 - k0 + STAGE - 1) / STAGE;

    // operands of the query rows: row 64 wq + 32 t + n, channels 16 s + 8 half ..
    uint4 qb[T][8];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int r = min(32 * T * wq + 32 * t + n, rows - 1);
        const uint16_t* qr = a.q + 8 * half;
        if constexpr (DRAFT) qr += (int64_t)(w.first * a.Hq + w.h * G + tables.row[r]) * HATA_D;
        else qr += ((int64_t)(w.first + r / G) * a.Hq + w.h * G + r % G) * HATA_D;
#pragma unroll
        for (int s = 0; s < 8; ++s) qb[t][s] = *reinterpret_cast<const uint4*>(qr + 16 * s);
    }
    float scale = fabsf(a.scale_log2);
    if constexpr (DRAFT) {
        if (scale == 0.f) {  // (the scores of rows that are not seen are -inf, and stay that)
            scale = 1.f;
#pragma unroll
            for (int t = 0; t < T; ++t)
#pragma unroll
                for (int s = 0; s < 8; ++s) qb[t][s] = make_uint4(0, 0, 0, 0);
        }
    }
    if (a.scale_log2 < 0.f) {  // (the maximum of the products is that of the scores then)
#pragma unroll
        for (int t = 0; t < T; ++t)
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
    auto first_row = [&](int s, int j) { return min(k0 + s * STAGE + wk * PART + (wq * BLOCKS + j) * 16, DRAFT ? (k1 - 1) & ~15 : k1 - 16); };
    auto look_up = [&](int s) {
#pragma unroll
        for (int j = 0; j < BLOCKS; ++j) pages[j] = table[first_row(s, j) >> a.pv.shift];
    };
    constexpr int FIRST = NBUF - (WQ > 1);  // stages requested before the first is waited for
    [[maybe_unused]] int first_pages[FIRST][BLOCKS];
    if constexpr (DRAFT) {
#pragma unroll
        for (int s = 0; s < FIRST; ++s)
#pragma unroll
            for (int j = 0; j < BLOCKS; ++j) first_pages[s][j] = table[first_row(s, j) >> a.pv.shift];
    } else {
        look_up(0);
    }
    // this wave's rows of a stage: PART wk + 16 BLOCKS wq + 16 j ..; lane l of an instruction fetches, of row 4 i + l / 16 of a block,
    // the piece that belongs at slot l % 16
    uint32_t off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) off[i] = (4 * i + (lane >> 4)) * 256 + ((lane & 15) ^ (lane >> 4 << 2 | i)) * 16;
    // (written as instructions: behind the compiler's builtin for it, every LDS read waits for all requests.  nt where the rows are read
    // by one tile of query rows, mostly: 12 sequences behind 131072 rows 119 -> 108 us, 32 behind 32768 68 -> 63; with eight tiles
    // it is the same, and slower where the caches hold the rows already.  Drafted tokens are one tile mostly: 32 sequences of 8192 rows with
    // 64 tokens 455 -> 449; 16 of 4096 with 256 tokens of 64 heads, eight tiles, 906 -> 918)
    auto fetch = [&](uint32_t dst, uint32_t o, const uint16_t* p) {
        if constexpr (WQ <= 2 || DRAFT)
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2 nt" ::"s"(dst), "v"(o), "s"(p) : "memory", "m0");
        else
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(dst), "v"(o), "s"(p) : "memory", "m0");
    };
    auto request = [&](int s, bool ahead = true) {
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
        if (ahead) look_up(s + 1);
    };
    // The sums and the query rows live in the accumulation registers, where the matrix instructions take them from, the scores in the
    // others; said at every turn, or the compiler moves the sums to and fro
    f32x16_t acc[T][4];
    float m[T], sub[T], l[T];
#pragma unroll
    for (int t = 0; t < T; ++t) { m[t] = HATA_NEG_INF; sub[t] = 0.f; l[t] = 0.f; }
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][c][i] = 0.f;
    auto pin = [&]() {
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int c = 0; c < 4; ++c) asm volatile("" : "+a"(acc[t][c]));
    };
    // K operand: row n, piece 2 s + half.  V operand: rows 16 x + 4 half + 8 y + (lane % 16) / 4, channels 32 c + lane's 16 and the
    // four of lane % 4
    const uint32_t k_at = n * 256 + ((half ^ prefix_swizzle(n)) << 4);
    const int v_row = 4 * half + (lane & 15) / 4, v_piece = (lane >> 4 & 1) * 2 + ((lane & 3) >> 1);

    auto products = [&](const char* kt, f32x16_t (&sc)[T]) {
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[t][i] = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const bf16x8_t kf = __builtin_bit_cast(bf16x8_t, *reinterpret_cast<const uint4*>(kt + (k_at ^ (k << 5))));
#pragma unroll
            for (int t = 0; t < T; ++t)
                sc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, __builtin_bit_cast(bf16x8_t, qb[t][k]), sc[t], 0, 0, 0);
        }
#pragma unroll
        for (int t = 0; t < T; ++t) asm volatile("" : "+v"(sc[t]));
    };
    auto highest = [&](const f32x16_t (&sc)[T], float (&top)[T]) {
#pragma unroll
        for (int t = 0; t < T; ++t) {
            top[t] = sc[t][0];
#pragma unroll
            for (int i = 1; i < 16; ++i) top[t] = fmaxf(top[t], sc[t][i]);
            top[t] *= scale;
        }
    };
    // the references, where the highest scores pass one
    auto follow = [&](const float (&top)[T]) {
        if (__builtin_amdgcn_ballot_w64(top[0] > m[0] || top[T - 1] > m[T - 1]) != 0ull) {
#pragma unroll
            for (int t = 0; t < T; ++t) {
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
    auto weights = [&](const f32x16_t (&sc)[T], uint32_t (&p)[2][T][8]) {
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = fast_exp2(fmaf(sc[t][2 * i], scale, -sub[t])), y = fast_exp2(fmaf(sc[t][2 * i + 1], scale, -sub[t]));
                p[0][t][i] = prefix_high(x, y);
                p[1][t][i] = prefix_low(x, y);
                l[t] = dot2_bf16(p[1][t][i], 0x3f803f80u, dot2_bf16(p[0][t][i], 0x3f803f80u, l[t]));
            }
    };
    auto values = [&](const char* vt, const uint32_t (&p)[2][T][8]) {
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
                    for (int t = 0; t < T; ++t)
                        acc[t][c] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            vf, __builtin_bit_cast(bf16x8_t, make_uint4(p[k][t][4 * x], p[k][t][4 * x + 1], p[k][t][4 * x + 2], p[k][t][4 * x + 3])), acc[t][c], 0, 0, 0);
            }
    };
    // ---- drafted rows ----
    [[maybe_unused]] __shared__ uint32_t s_bad[8];  // drafted rows with values that are not finite
    // Scores of 32 rows, the stage's from `from` on, that a query row does not see, or that are not there: -inf
    [[maybe_unused]] auto hide = [&](int s, int from, f32x16_t (&sc)[T]) {
        const int r0 = k0 + s * STAGE + from, d = r0 - base;
#pragma unroll
        for (int t = 0; t < T; ++t) {
            const uint32_t* bits = tables.seen + tables.member[32 * T * wq + 32 * t + n] * SEEN_WORDS;  // (of a member that is not there: anything)
            uint32_t see = 0;
            if (d < 0) see = d <= -32 ? ~0u : ((1u << -d) - 1) | bits[0] << -d;
            else if (d < 256) see = (uint32_t)(((unsigned long long)bits[(d >> 5) + 1] << 32 | bits[d >> 5]) >> (d & 31));
            see >>= 4 * half;
#pragma unroll
            for (int i = 0; i < 16; ++i) sc[t][i] = see >> (8 * (i / 4) + i % 4) & 1 ? sc[t][i] : HATA_NEG_INF;
        }
    };
    // Values that a weight of zero would not keep out: rows that are not there, and of drafted ones those that are not finite
    [[maybe_unused]] auto clean = [&](int s, int from, int at, int step, int count) {
        char* vt = smem + (s % NBUF) * STAGE * 512 + STAGE * 256 + from * 256;
        for (int e = at; e < count * 16; e += step) {
            const int row = k0 + s * STAGE + from + e / 16;
            if (row < base) continue;
            uint4* p = reinterpret_cast<uint4*>(vt + e * 16);
            if (row >= end) { *p = make_uint4(0, 0, 0, 0); continue; }
            uint4 v = *p;
            bool bad = false;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                uint32_t& x = (&v.x)[i];
                const bool lo = (x & 0x7f80u) == 0x7f80u, hi = (x & 0x7f800000u) == 0x7f800000u;
                bad |= lo | hi;
                x &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
            }
            if (bad) {
                *p = v;
                atomicOr(&s_bad[(row - base) >> 5], 1u << ((row - base) & 31));
            }
        }
        if (step == 64) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // (of this wave alone)
    };
    // ... which those that see the row have in their sums as they are, whatever the weight
    [[maybe_unused]] auto add_bad = [&]() {
        for (int k = 0; k < 8; ++k)
            for (uint32_t rows_left = s_bad[k]; rows_left; rows_left &= rows_left - 1) {
                const int j = 32 * k + __ffs(rows_left) - 1, row = base + j;
                const int page = clampi(table[row >> a.pv.shift], 0, a.pv.n_pages - 1);
                const uint16_t* v = a.V + ((((int64_t)page * a.Hkv + w.h) << a.pv.shift) + (row & ((1 << a.pv.shift) - 1))) * HATA_D;
#pragma unroll
                for (int t = 0; t < T; ++t) {
                    const bool sees = tables.seen[tables.member[32 * T * wq + 32 * t + n] * SEEN_WORDS + k] >> (j & 31) & 1;
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float x = __uint_as_float((uint32_t)v[32 * c + 8 * (i / 4) + 4 * half + i % 4] << 16);
                            acc[t][c][i] += sees && !(fabsf(x) < __builtin_huge_valf()) ? x : 0.f;
                        }
                }
            }
    };
    if constexpr (DRAFT) {
        if (tid < 8) s_bad[tid] = 0;
        __syncthreads();
    }
    auto at_stage = [&](int s) { return (const char*)smem + (s % NBUF) * STAGE * 512 + wk * PART * 256; };  // K; V is STAGE * 256 bytes behind

    // (the wait for the query rows is one for every request so far: the first stage's only)
    if constexpr (!DRAFT) request(0);
#pragma unroll
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int s = 0; s < 8; ++s)  // (used here, so that the wait for these loads is not in the loop)
            asm volatile("" : "+a"(qb[t][s].x), "+a"(qb[t][s].y), "+a"(qb[t][s].z), "+a"(qb[t][s].w));
    pin();
    // (with several query waves a stage behind the last one is the last rows once more: as many requests are outstanding everywhere)
    if constexpr (DRAFT) {  // (their pages are looked up together, beside the query rows)
#pragma unroll
        for (int s = 0; s < FIRST; ++s)
            if (WQ > 1 || s < stages) {
#pragma unroll
                for (int j = 0; j < BLOCKS; ++j) pages[j] = first_pages[s][j];
                request(s, s + 1 == FIRST);
            }
    } else {
        for (int s = 1; s < NBUF - (WQ > 1); ++s)
            if (WQ > 1 || s < stages) request(s);
    }
    if constexpr (WQ == 1) {
        // rows of this wave alone: nothing is waited for but its own requests
        for (int s = 0; s < stages; ++s) {
            if (s + 1 < stages) prefix_wait<BLOCKS * 8>();
            else prefix_wait<0>();
            if (k0 + s * STAGE + wk * PART < k1) {
                f32x16_t sc[T];
                uint32_t p[2][T][8];
                float top[T];
                products(at_stage(s), sc);
                if constexpr (DRAFT) {
                    if (k0 + s * STAGE + wk * PART + 32 > base) {
                        hide(s, wk * PART, sc);
                        clean(s, wk * PART, lane, 64, PART);
                    }
                }
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
        if constexpr (DRAFT) {
            if (k0 + STAGE > base) {
                clean(0, 0, tid, 256, STAGE);
                __syncthreads();
            }
        }
        bool idle = false;
        if constexpr (DRAFT) idle = 64 * wq >= rows;
        if (idle) {  // (no query rows: this wave's requests and barriers alone)
            for (int s = 0; s < stages; ++s) {
                prefix_wait<(NBUF - 3) * 8>();
                __syncthreads();
                if (s + 1 < stages && k0 + (s + 2) * STAGE > base) {
                    clean(s + 1, 0, tid, 256, STAGE);
                    __syncthreads();
                }
                request(s + NBUF - 1);
            }
        } else {
            products(at_stage(0), sc);
            highest(sc, top);
        }
        for (int s = 0; s < (idle ? 0 : stages); ++s) {
#pragma unroll
            for (int i = 0; i < SUBS; ++i) {
                uint32_t p[2][2][4];  // [turn and turn][query row][two rows]
                if constexpr (DRAFT) {
                    if (k0 + s * STAGE + wk * PART + (i + 1) * 32 > base) {
                        hide(s, wk * PART + i * 32, sc);
                        highest(sc, top);
                    }
                }
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
                    if constexpr (DRAFT) {
                        if (s + 1 < stages && k0 + (s + 2) * STAGE > base) {
                            clean(s + 1, 0, tid, 256, STAGE);
                            __syncthreads();
                        }
                    }
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
                for (int t = 0; t < T; ++t)
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
                for (int t = 0; t < T; ++t) sc[t] = next[t];
                pin();
            }
        }
    }

    // ---- the waves' sums, joined where they have the same query rows ----
    prefix_wait<0>();
    __syncthreads();  // the ring is no longer read
    if constexpr (DRAFT) {
        if (wk == 0 && k1 > base) add_bad();
    }
    float* s_acc = reinterpret_cast<float*>(smem);  // [wave][64][HATA_D + 4]
    __shared__ float s_m[4][64], s_l[4][64];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        float x, y;
        swap32(l[t], x, y);
        l[t] = x + y;
        if (half == 0) { s_m[wave][32 * t + n] = m[t]; s_l[wave][32 * t + n] = l[t]; }
    }
    float top[T], total[T];
#pragma unroll
    for (int t = 0; t < T; ++t) { top[t] = m[t]; total[t] = l[t]; }
    if constexpr (WK > 1) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < T; ++t) {
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
    for (int t = 0; t < T; ++t)
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)  // acc[t][c][4 i + j]: channel 32 c + 8 i + 4 half + j of query row 32 t + n
                *reinterpret_cast<float4*>(&s_acc[(wave * 64 + 32 * t + n) * (HATA_D + 4) + 32 * c + 8 * i + 4 * half]) =
                    make_float4(acc[t][c][4 * i], acc[t][c][4 * i + 1], acc[t][c][4 * i + 2], acc[t][c][4 * i + 3]);
    [[maybe_unused]] __shared__ float s_inverse[M];
    if constexpr (DRAFT) {
        if (wk == 0 && half == 0) {
#pragma unroll
            for (int t = 0; t < T; ++t) s_inverse[32 * T * wq + 32 * t + n] = total[t] == 0.f ? 0.f : 1.f / total[t];
        }
    }
    __syncthreads();
    bool final = false;
    int part_rows = M;
    if constexpr (DRAFT) {
        final = w.final;
        part_rows = a.part_rows;
    }
    float* out = a.part + (int64_t)w.item * (part_rows * (HATA_D + 2));
    if (!final && wk == 0 && half == 0) {
#pragma unroll
        for (int t = 0; t < T; ++t)
            if (64 * wq + 32 * t + n < rows)
                *reinterpret_cast<float2*>(out + part_rows * HATA_D + 2 * (64 * wq + 32 * t + n)) = make_float2(top[t], total[t]);
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
        if constexpr (DRAFT) {
            if (final) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = i0 + 8 * j + r8;
                    if (r >= rows) continue;
                    const float f = s_inverse[r];
                    // (no weight at all: zeros, also where a value that is not finite made the sums NaN)
                    o[j] = f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[j].x * f, o[j].y * f, o[j].z * f, o[j].w * f);
                    store_output(a.out, a.out_f32, (int64_t)(w.first * a.Hq + w.h * G + tables.row[r]) * HATA_D + c4, o[j]);
                }
                continue;
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (i0 + 8 * j + r8 < rows) *reinterpret_cast<float4*>(out + (i0 + 8 * j + r8) * HATA_D + c4) = o[j];
    }
}

}  // namespace hata
