// Pages of a paged cache: block tables and slot maps from request lengths, and packed rows written through a slot map.
#include <algorithm>
#include "hata_attn_core.h"
#include "hata_device.h"
#include "hata_encode_core.h"
#include "hata_hash.h"
#include "hata_internal.h"

namespace hata {

// ---- block tables and slot map (hata_plan_pages) ----
//
// With blocks(n) = ceil(n / page_rows), sequence b needs need[b] = max(0, blocks(next) - blocks(now)) pages and, where it
// shrinks, releases the blocks from max(blocks(next), shared) up to blocks(now).  Page j of all that are needed, in the order of
// the sequences, is number avail - 1 - j of the free list with the released pages behind it (avail: their sum), so that
// neither the tables nor the list need an exchange between workgroups: a page that is released and taken in the same call is
// looked up in the table that releases it.  Written are rows of growing sequences and list entries from n_free on, read are
// rows of shrinking sequences and list entries below n_free.  What every workgroup reads and the caller may have given as an
// output too (lengths, n_free) is written by the last workgroup to arrive.
// Bound by latency: launch, lengths, sums, a page, a slot, one after the other.  32 sequences of a token each 5.9 us; 704 sequences
// with 198779 new rows 12.7 (one workgroup 1690; 256 of them 16.5, a counter for all 512 17.6, pages behind the slots 17).
// (uint32_t sums: HATA_PLAN_MAX_B sequences of 2^19 blocks, the most an L_cap of 2^23 rows has)
#define PLAN_THREADS 256
#define PLAN_BATCH 4
#define PLAN_TOKENS_SAT ((1u << 23) + 1)  // above every max_tokens; 256 of them still are a 32-bit number

struct PlanRequest {
    int now, next, src;  // rows cached and wanted, clamped at 0; the sequence that is forked, or -1
    int have, want, keep, n_new;
    bool valid;          // the sums left aside
};

__device__ __forceinline__ PlanRequest plan_request(const PagePlan& p, int b) {
    PlanRequest r;
    const int P1 = (1 << p.shift) - 1;
    const int now = p.len_now[b], next = p.len_next[b];
    r.src = p.fork_from ? p.fork_from[b] : -1;
    r.valid = now >= 0 && next >= 0 && now <= p.cap && next <= p.cap;
    r.now = max(now, 0);
    r.next = max(next, 0);
    r.n_new = max(r.next - r.now, 0);
    r.have = (min(r.now, p.cap) + P1) >> p.shift;
    r.want = (min(r.next, p.cap) + P1) >> p.shift;
    r.keep = max(r.want, p.shared_blocks ? p.shared_blocks[b] : 0);
    if (r.src >= 0) {
        const int s = min(r.src, p.B - 1);
        const int held = min(min(p.len_now[s], p.len_next[s]), p.cap) >> p.shift;  // whole pages the source keeps
        r.valid = r.valid && r.src < p.B && r.src != b && p.fork_from[s] < 0 && (r.now & P1) == 0 && r.next >= r.now &&
                  r.now >> p.shift <= held;
    }
    return r;
}

// sums over the workgroup's threads below this one
__device__ __forceinline__ uint32_t plan_before(uint32_t v, uint32_t* lds4) {
    uint32_t total;
    return block_excl_scan_256(v, lds4, &total);
}

__global__ __launch_bounds__(PLAN_THREADS) void plan_pages_kernel(const PagePlan p, uint32_t* counter) {
    extern __shared__ uint32_t plan_lds[];
    __shared__ uint32_t lds4[4];
    __shared__ int s_last;
    uint32_t* tok_end = plan_lds;         // [B] packed rows up to and with sequence b's, at most PLAN_TOKENS_SAT; top bit: the request is valid and its rows fit
    uint32_t* need_end = tok_end + p.B;   // [B] the same for the pages that are needed
    uint32_t* gone_end = need_end + p.B;  // [B] for the pages that are released
    uint32_t* copy_end = gone_end + p.B;  // [B] for the blocks that forks copy
    const int tid = threadIdx.x, B = p.B;
    const int n_free = clampi(*p.n_free, 0, p.n_pages);
    constexpr uint32_t OK = 0x80000000u;
    // what every request adds, read side by side; then the sums, a run of sequences a thread
#pragma unroll 4
    for (int b = tid; b < B; b += PLAN_THREADS) {
        const PlanRequest r = plan_request(p, b);
        tok_end[b] = (uint32_t)min(r.n_new, 1 << 23) | (r.valid ? OK : 0u);
        need_end[b] = (uint32_t)max(r.want - r.have, 0);
        gone_end[b] = r.next < r.now ? (uint32_t)max(r.have - r.keep, 0) : 0u;
        copy_end[b] = r.src >= 0 ? (uint32_t)(r.now >> p.shift) : 0u;
    }
    __syncthreads();
    {
        const int per = (B + PLAN_THREADS - 1) / PLAN_THREADS, b0 = min(tid * per, B), b1 = min(b0 + per, B);
        uint32_t sum = 0, need = 0, gone = 0, copy = 0;
        for (int b = b0; b < b1; ++b) sum += tok_end[b] & ~OK;
        uint32_t at = plan_before(min(sum, PLAN_TOKENS_SAT), lds4);
        for (int b = b0; b < b1; ++b) {
            const uint32_t own = tok_end[b] & ~OK, end = min(at += own, PLAN_TOKENS_SAT);
            const bool ok = (tok_end[b] & OK) && (own == 0 || end <= (uint32_t)p.max_tokens);
            tok_end[b] = end | (ok ? OK : 0u);
            need_end[b] = need += ok ? need_end[b] : 0u;
            gone_end[b] = gone += ok ? gone_end[b] : 0u;
            copy_end[b] = copy += ok ? copy_end[b] : 0u;
        }
        need = plan_before(need, lds4);
        gone = plan_before(gone, lds4);
        copy = plan_before(copy, lds4);
        for (int b = b0; b < b1; ++b) {
            need_end[b] += need;
            gone_end[b] += gone;
            copy_end[b] += copy;
        }
    }
    __syncthreads();
    const uint32_t all_gone = gone_end[B - 1], all_need = need_end[B - 1], all_copy = copy_end[B - 1];
    const uint32_t all_tokens = tok_end[B - 1] & ~OK;
    const int64_t avail = (int64_t)n_free + all_gone;
    auto value = [&](const uint32_t* end, int b) { return end == tok_end ? end[b] & ~OK : end[b]; };
    auto before = [&](const uint32_t* end, int b) { return b ? value(end, b - 1) : 0u; };
    auto granted = [&](int b) {
        const uint32_t to = need_end[b];
        return (tok_end[b] & OK) && (to == before(need_end, b) || (int64_t)to <= avail);
    };
    // the first sequence whose sum is above i
    auto find = [&](const uint32_t* end, uint32_t i) {
        int lo = 0, n = B;
        while (n > 1) {
            const int half = n / 2;
            if (value(end, lo + half - 1) <= i) { lo += half; n -= half; }
            else n = half;
        }
        return lo;
    };
    // pages taken: those up to the last sequence that gets what it needs
    uint32_t used = all_need;
    if ((int64_t)all_need > avail) {
        // (the sums grow: the last one not above avail)
        const int b = find(need_end, (uint32_t)avail);  // need_end[b] > avail
        used = before(need_end, b);
    }
    const int64_t left = avail - used;
    auto released_at = [&](uint32_t i) -> const int32_t* {  // where page number i of those released is found
        const int b = find(gone_end, i);
        const int P1 = (1 << p.shift) - 1, want = (p.len_next[b] + P1) >> p.shift;
        const int keep = max(want, p.shared_blocks ? p.shared_blocks[b] : 0);
        return p.table + (int64_t)b * p.max_blocks + keep + (int)(i - before(gone_end, b));
    };
    auto taken_at = [&](uint32_t j) -> const int32_t* {  // page number j of those needed
        const int64_t i = avail - 1 - j;
        return i >= n_free ? released_at((uint32_t)(i - n_free)) : p.free_pages + i;
    };
    auto page_number = [&](int v) { return clampi(v, 0, p.n_pages - 1); };
    // Slots by the first workgroups, pages by the others, a chain of look-ups each: one behind the other they took twice as long.
    // PLAN_BATCH elements of a thread go through a chain together.
    const int slot_wgs = gridDim.x < 4 ? (int)gridDim.x : (int)(gridDim.x - gridDim.x / 4);
    const bool pages_too = gridDim.x < 4, slot_wg = (int)blockIdx.x < slot_wgs;
    if (slot_wg) {
        const uint32_t step = (uint32_t)slot_wgs * PLAN_THREADS;
        for (uint32_t t = blockIdx.x * PLAN_THREADS + tid; t < (uint32_t)p.max_tokens; t += step) {
            int slot = -1, pos = -1;
            if (t < all_tokens) {
                const int b = find(tok_end, t);
                if (granted(b)) {
                    const int now = p.len_now[b], P1 = (1 << p.shift) - 1, have = (now + P1) >> p.shift;
                    pos = now + (int)(t - before(tok_end, b));
                    const int block = pos >> p.shift;
                    const int32_t* at = block < have ? p.table + (int64_t)b * p.max_blocks + block
                                                     : taken_at(before(need_end, b) + (uint32_t)(block - have));
                    slot = (page_number(*at) << p.shift) + (pos & P1);
                }
            }
            p.slots[t] = slot;
            if (p.positions) p.positions[t] = pos;
        }
    }
    if (!slot_wg || pages_too) {
        // a wave per sequence
        const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        const int first = (int)(pages_too ? blockIdx.x : blockIdx.x - slot_wgs) * 4 + wave;
        const int step = (int)(pages_too ? gridDim.x : gridDim.x - slot_wgs) * 4;
        const int64_t spare = min(left, (int64_t)p.n_pages) - n_free;  // released pages that nobody took
        // n elements, element i read at src + i and written to dst + i
        auto move = [&](const int32_t* src, int32_t* dst, int n) {
            for (int i0 = lane; i0 < n; i0 += 64 * PLAN_BATCH) {
                int v[PLAN_BATCH];
#pragma unroll
                for (int k = 0; k < PLAN_BATCH; ++k) v[k] = src[min(i0 + 64 * k, n - 1)];
#pragma unroll
                for (int k = 0; k < PLAN_BATCH; ++k)
                    if (i0 + 64 * k < n) dst[i0 + 64 * k] = v[k];
            }
        };
        for (int b = first; b < B; b += step) {
            const uint32_t need0 = before(need_end, b), gone0 = before(gone_end, b), copy0 = before(copy_end, b);
            const int need = (int)(need_end[b] - need0), gone = (int)(gone_end[b] - gone0), copy = (int)(copy_end[b] - copy0);
            if ((need | gone | copy) == 0 || !granted(b)) continue;
            int32_t* row = p.table + (int64_t)b * p.max_blocks;
            const int P1 = (1 << p.shift) - 1, have = (p.len_now[b] + P1) >> p.shift;
            for (int i = lane; i < need; i += 64) row[have + i] = page_number(*taken_at(need0 + i));
            if (copy) move(p.table + (int64_t)p.fork_from[b] * p.max_blocks, row, copy);
            if (gone) move(row + (have - gone), p.free_pages + n_free + gone0, (int)min((int64_t)gone, max(spare - (int64_t)gone0, (int64_t)0)));
        }
    }
    if (gridDim.x > 1) {
        __syncthreads();  // nothing of this workgroup reads lengths or n_free after this
        if (tid == 0) {
            // (in groups: arrivals at one counter come 17 ns apart)
            const int group = blockIdx.x / HATA_PLAN_GROUP, groups = (gridDim.x + HATA_PLAN_GROUP - 1) / HATA_PLAN_GROUP;
            uint32_t* own = counter + (1 + group) * HATA_COUNTER_STRIDE;
            int last = atomicAdd(own, 1u) == min(HATA_PLAN_GROUP, (int)gridDim.x - group * HATA_PLAN_GROUP) - 1;
            if (last) {
                *own = 0;
                last = atomicAdd(counter, 1u) == groups - 1;
                if (last) *counter = 0;
            }
            s_last = last;
        }
        __syncthreads();
        if (!s_last) return;
    } else {
        __syncthreads();
    }
    for (int b = tid; b < B; b += PLAN_THREADS) {
        const int now = clampi(p.len_now[b], 0, p.cap), next = p.len_next[b];
        const int forked = p.fork_from && p.fork_from[b] >= 0;
        p.seq_len[b] = granted(b) ? next : forked ? 0 : now;
        if (p.token_start) p.token_start[b] = (int)min(before(tok_end, b), (uint32_t)p.max_tokens);
    }
    if (tid == 0) {
        if (p.token_start) p.token_start[B] = (int)min(all_tokens, (uint32_t)p.max_tokens);
        *p.n_free_out = (int)min(left, (int64_t)p.n_pages);
    }
}

hipError_t prepare_pages() {  // (more than 64 KB of dynamic LDS has to be asked for)
    return hipFuncSetAttribute((const void*)plan_pages_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, HATA_PLAN_MAX_B * 16);
}

hipError_t launch_plan_pages(const hata_ctx* c, const PagePlan& p, hipStream_t s) {
    const int wgs = std::max(1, std::min(HATA_PLAN_WGS, std::max((p.max_tokens + PLAN_THREADS - 1) / PLAN_THREADS, p.B / 4)));
    hipLaunchKernelGGL(plan_pages_kernel, dim3(wgs), dim3(PLAN_THREADS), (size_t)p.B * 16, s, p, c->plan_counter);
    return hipGetLastError();
}

// ---- packed rows into pages (hata_write_slots) ----
//
// grid = (slices of COLS hash columns, Hkv, runs of WRITE_ROWS packed rows); the first slice copies the rows.  Codes in fp64
// (hata_hash.h), four rows at a time.
#define WRITE_ROWS 16
// Rows up to which a call with codes goes this way: us, eight heads, r = 128, this way / by the matrix cores with prepared weights / without:
// 64 rows 6.3 / 6.2 / 9.4, 128 6.3 / 6.4 / 9.5, 256 6.5 / 6.6 / 9.8, 512 9.2 / 6.9 / 9.9, 1024 14.7 / 7.6 / 10.4; r = 256, 64 6.2 / 7.0 / 12.0,
// 128 6.5 / 7.3 / 12.4, 256 9.2 / 7.5 / 12.4, 512 14.8 / 8.6 / 13.0.  (One number for both: a server's weights are fixed, and prepared; without
// that, 129 to some 400 rows take up to 4 us longer than they would this way.)  Widths other than 32, 64, 128 and 256 go this way at any
// number of rows: no configuration here has one.  20711 rows, r = 96: 286 us.
#define HATA_WRITE_FEW 128
struct WriteSlots {
    const uint16_t *K_new, *V_new;
    const int32_t* slots;
    uint16_t *K, *V;
    uint32_t* codes;
    const float* W_H;
    int64_t st, sh;
    int n, Hkv, r, shift, rows;  // rows: of one head in the pools
};

__device__ __forceinline__ int64_t slot_row(const WriteSlots& a, int slot, int h) {
    return (((int64_t)(slot >> a.shift) * a.Hkv + h) << a.shift) + (slot & ((1 << a.shift) - 1));
}

template <int COLS>
__global__ __launch_bounds__(256) void write_few_kernel(const WriteSlots a) {
    constexpr int WPS = COLS / 32;
    __shared__ uint32_t s_codes[(WRITE_ROWS + 4) * WPS];
    const int tid = threadIdx.x, h = blockIdx.y, t0 = blockIdx.z * WRITE_ROWS, nv = min(WRITE_ROWS, a.n - t0);
    if (blockIdx.x == 0) {
        const int t = t0 + (tid >> 4), o = (tid & 15) * 8;
        const int slot = t < a.n ? a.slots[t] : -1;
        if (slot >= 0 && slot < a.rows) {
            const int64_t from = t * a.st + h * a.sh + o, to = slot_row(a, slot, h) * HATA_D + o;
            *reinterpret_cast<uint4*>(a.K + to) = *reinterpret_cast<const uint4*>(a.K_new + from);
            *reinterpret_cast<uint4*>(a.V + to) = *reinterpret_cast<const uint4*>(a.V_new + from);
        }
    }
    if (!a.codes) return;
    HashWeights<COLS> hw;
    hw.fetch(a.W_H + (int64_t)h * HATA_D * a.r + blockIdx.x * COLS, a.r);
    for (int v0 = 0; v0 < nv; v0 += 4) {
        uint4 x[4];
        hash_load_x(a.K_new + (int64_t)(t0 + min(v0 + (tid & 3), nv - 1)) * a.st + h * a.sh, x);
        hash_pass<COLS>(hw, x, s_codes, WPS, v0, nv);
    }
    __syncthreads();
    for (int i = tid; i < nv * WPS; i += 256) {
        const int slot = a.slots[t0 + i / WPS];
        if (slot >= 0 && slot < a.rows) a.codes[slot_row(a, slot, h) * (a.r / 32) + blockIdx.x * WPS + i % WPS] = s_codes[i];
    }
}

// Many rows: the projection on the matrix cores, as in encode_mfma_kernel (M = 32 hash columns of a wave, N = 32 rows; prepared
// fp16 planes, or three bf16 planes split here), and the values next to zero once more in fp64.
//
// A sum of the matrix cores is within half of WRITE_ERROR |x| |w| of the exact one (Euclidean norms; at most 24 instructions, each off by a
// few units in the last place of a partial sum, which |x| |w| bounds).  A sum that is not above the whole (one value in some 7000 of
// normally distributed ones) is in doubt: it goes on a list, and once the workgroup is through its rows, each of them is evaluated as
// fewer rows are (hash_pass): in fp64, where the products are exact, with the same roundings of the sums.  So a key's code does not
// depend on the number of rows, not even where its products cancel further than fp64 reaches.  (Evaluated where they were found, by a wave each, they cost a latency a stage.
// 20711 rows, eight heads, r = 128, us: 46.0 that way, 38.2 with the list by sixteen lanes of the vector ALU an item, 37.2 as here.)
// fp16 planes: x loses up to 2^-24 below 2^-14 and saturates at 65504, the weights 2^-22 of their size or 2^-25; rows of which that
// says nothing, because they are as large or as small as the numbers get, infinite or NaN, are evaluated in fp64 as a whole.
//
// Bound by the bytes it moves (512 read and 512 written a row), then by the products, which do not overlap with them on this
// device: those 20711 rows 37.2 us, 4.65 TB/s, where a large copy reaches 4.8; 16384 rows of 32 heads, r = 256, 144 us, 3.9 TB/s.  (Three planes, split
// here by every workgroup, where the weights are not prepared: 42.9 and 168 us.)
// Rounds of resident workgroups (write_rows_per_wg): 45.4 us with twice as many of half the rows.
#define WRITE_ERROR 0x1p-16f
#define WRITE_MAX_ROWS 1024  // of a workgroup
#define WRITE_DOUBTS 512
template <int R, bool F16>
__global__ __launch_bounds__(R <= 128 ? 256 : 512, 2) void write_mfma_kernel(const WriteSlots a, const uint4* __restrict__ planes, int rows_per_wg) {
    constexpr int COLW = R / 32, KP = R >= 128 ? 1 : 128 / R;  // waves by columns, by rows
    constexpr int THREADS = 64 * COLW * KP, NT = R >= 128 ? 2 : 1, STAGE = 32 * NT * KP, WD = R / 32;
    constexpr int ROWS_PER_IT = THREADS / 16, NIT = STAGE / ROWS_PER_IT;
    __shared__ __attribute__((aligned(16))) uint16_t tile[STAGE * HATA_MFMA_PITCH];
    __shared__ __attribute__((aligned(16))) uint32_t s_code[WRITE_MAX_ROWS * WD];
    __shared__ float s_norm[STAGE];
    __shared__ int s_row[WRITE_MAX_ROWS];
    __shared__ uint32_t s_doubt[WRITE_DOUBTS];  // row of the workgroup * R + column
    __shared__ int s_doubts, s_wholes;
    __shared__ uint32_t s_whole[WRITE_MAX_ROWS / 32];  // rows of which every bit is in doubt
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int w = wave % COLW, part = wave / COLW, m = lane & 31, half = lane >> 5, h = blockIdx.y;
    const int first = blockIdx.x * rows_per_wg, last = min(first + rows_per_wg, a.n);
    const uint16_t* Kh = a.K_new + h * a.sh;
    const uint16_t* Vh = a.V_new + h * a.sh;

    const int lrow = tid >> 4, lsub = tid & 15;
    uint4 pre[NIT], vpre[NIT];
    int slot[NIT];
    auto load_stage = [&](int t0) {
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
            const int t = t0 + it * ROWS_PER_IT + lrow;
            slot[it] = a.slots[min(t, last - 1)];
            if (t >= last) slot[it] = -1;
        }
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
            const int64_t o = min(t0 + it * ROWS_PER_IT + lrow, last - 1) * a.st + lsub * 8;
            pre[it] = load_once(Kh + o);
            vpre[it] = load_once(Vh + o);
        }
    };
    load_stage(first);
    if (tid == 0) s_doubts = s_wholes = 0;
    if (tid < WRITE_MAX_ROWS / 32) s_whole[tid] = 0;

    // weight fragments, and the largest norm of this wave's columns (of the fp16 planes: scaled as they are)
    bf16x8_t afrag[F16 ? 1 : 3][F16 ? 1 : 8];
    f16x8_t afrag16[F16 ? 2 : 1][F16 ? 8 : 1];
    float norm2 = 0.f, some_w = 0.f;
    if constexpr (F16) {
        const uint4* src = planes + ((int64_t)(h * COLW + w) * 8 * 2) * 64 + lane;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
#pragma unroll
            for (int p = 0; p < 2; ++p) afrag16[p][kk] = __builtin_bit_cast(f16x8_t, src[(kk * 2 + p) * 64]);
#pragma unroll
            for (int e = 0; e < 8; ++e) norm2 = fmaf((float)afrag16[0][kk][e], (float)afrag16[0][kk][e], norm2);
        }
        some_w = norm2;  // (the largest weight of a tile is scaled to 2^13 or more)
    } else {
        const float* wp = a.W_H + (int64_t)h * HATA_D * R + w * 32 + m;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) {
            uint32_t hi[4], mid[4], lo[4];
#pragma unroll
            for (int e2 = 0; e2 < 4; ++e2) {
                const float w0 = wp[(int64_t)(kk * 16 + 8 * half + 2 * e2) * R], w1 = wp[(int64_t)(kk * 16 + 8 * half + 2 * e2 + 1) * R];
                split_weight_pair(w0, w1, hi[e2], mid[e2], lo[e2]);
                norm2 = fmaf(w0, w0, fmaf(w1, w1, norm2));
                some_w = fmaxf(some_w, fmaxf(fabsf(w0), fabsf(w1)));
            }
            afrag[0][kk] = __builtin_bit_cast(bf16x8_t, make_uint4(hi[0], hi[1], hi[2], hi[3]));
            afrag[1][kk] = __builtin_bit_cast(bf16x8_t, make_uint4(mid[0], mid[1], mid[2], mid[3]));
            afrag[2][kk] = __builtin_bit_cast(bf16x8_t, make_uint4(lo[0], lo[1], lo[2], lo[3]));
        }
    }
    norm2 += __shfl_xor(norm2, 32, 64);
    // (the maximum drops NaN; of tiny weights, whose squares are lost, all rows are evaluated in fp64)
    const bool doubt = __builtin_amdgcn_ballot_w64(!(norm2 < 0x1p120f)) != 0ull;
    norm2 = wave_max64(norm2);
    const bool no_w = !doubt && __builtin_amdgcn_ballot_w64(some_w != 0.f) == 0ull;
    const float wn = no_w ? 0.f : doubt || norm2 < 0x1p-80f ? __builtin_huge_valf() : sqrtf(norm2);

    for (int t0 = first; t0 < last; t0 += STAGE) {
        __syncthreads();  // the previous stage has been consumed
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
            const int row = it * ROWS_PER_IT + lrow;
            const uint4 x = pre[it];
            *reinterpret_cast<uint4*>(&tile[row * HATA_MFMA_PITCH + lsub * 8]) = F16 ? __builtin_bit_cast(uint4, bf16x8_to_f16(x)) : x;
            const float n2 = row_sum16(dot2_bf16(x.x, x.x, dot2_bf16(x.y, x.y, dot2_bf16(x.z, x.z, dot2_bf16(x.w, x.w, 0.f)))));
            const float some = row_max16(((x.x | x.y | x.z | x.w) & 0x7fff7fffu) ? 1.f : 0.f);
            int to = -1;
            if (slot[it] >= 0 && slot[it] < a.rows) {
                to = (int)slot_row(a, slot[it], h);
                *reinterpret_cast<uint4*>(a.K + (int64_t)to * HATA_D + lsub * 8) = x;
                *reinterpret_cast<uint4*>(a.V + (int64_t)to * HATA_D + lsub * 8) = vpre[it];
            }
            if (lsub == 0) {
                // (a row of zeros projects to zero, in any arithmetic that holds the weights, and so does a finite row where they are zeros)
                const bool in_range = n2 < (F16 ? 0x1p31f : 0x1p120f) && (n2 >= 0x1p-80f || some == 0.f);
                s_norm[row] = in_range ? sqrtf(n2) : __builtin_huge_valf();
                s_row[t0 - first + row] = to;
            }
        }
        __syncthreads();
        if (t0 + STAGE < last) load_stage(t0 + STAGE);  // overlaps the products below

        f32x16_t acc[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[t][i] = 0.f;
        const int row0 = part * 32 * NT;
        uint4 bfrag[NT];  // (a channel step ahead)
#pragma unroll
        for (int t = 0; t < NT; ++t) bfrag[t] = *reinterpret_cast<const uint4*>(&tile[(row0 + t * 32 + m) * HATA_MFMA_PITCH + 8 * half]);
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                if constexpr (F16) {
#pragma unroll
                    for (int p = 0; p < 2; ++p)
                        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_f16(afrag16[p][kk], __builtin_bit_cast(f16x8_t, bfrag[t]), acc[t], 0, 0, 0);
                } else {
#pragma unroll
                    for (int p = 0; p < 3; ++p)
                        acc[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(afrag[p][kk], __builtin_bit_cast(bf16x8_t, bfrag[t]), acc[t], 0, 0, 0);
                }
                if (kk + 1 < 8)
                    bfrag[t] = *reinterpret_cast<const uint4*>(&tile[(row0 + t * 32 + m) * HATA_MFMA_PITCH + (kk + 1) * 16 + 8 * half]);
            }
        // this lane holds hash columns 8 (i / 4) + 4 half + i % 4 of row t * 32 + m
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            uint32_t word = sign_bits(acc[t]);
            const int row = row0 + t * 32 + m;
            const float xn = s_norm[row], near = F16 ? wn * fmaf(WRITE_ERROR, xn, 0x1p-20f) + 0x1p-21f * xn : WRITE_ERROR * wn * xn;
            float least = fabsf(acc[t][0]);
#pragma unroll
            for (int i = 1; i < 16; ++i) least = fminf(least, fabsf(acc[t][i]));
            const bool zeros = (xn == 0.f && wn < __builtin_huge_valf()) || wn == 0.f;  // (weights out of range may be infinite in the planes)
            const bool live = s_row[t0 - first + row] >= 0;
            if (__builtin_amdgcn_ballot_w64(live && !zeros && !(least > near)) != 0ull) {
                uint32_t todo = 0;
#pragma unroll
                for (int i = 0; i < 16; ++i) todo |= (!(fabsf(acc[t][i]) > near) ? 1u : 0u) << (8 * (i / 4) + i % 4);
                if (zeros || !live) todo = 0;
                const int r = t0 - first + row;
                bool whole = todo != 0 && !(near < __builtin_huge_valf());
                for (; todo && !whole; todo &= todo - 1) {
                    const int at = atomicAdd(&s_doubts, 1);
                    whole = at >= WRITE_DOUBTS;  // (no room)
                    if (!whole) s_doubt[at] = (uint32_t)r * R + 32 * w + 4 * half + __ffs(todo) - 1;
                }
                if (whole) {
                    atomicOr(&s_whole[r / 32], 1u << (r % 32));
                    s_wholes = 1;
                }
            }
            word <<= 4 * half;
            word |= (uint32_t)__shfl_xor((int)word, 32, 64);
            if (half == 0) s_code[(t0 - first + row) * WD + w] = word;
        }
    }
    __syncthreads();
    // Bits in doubt, sixteen a wave: hash_pass' instruction and its order of the channels, so that the sums round as they do there.  Its
    // four blocks take four columns and four vectors each, of which the diagonal is looked at: lane l has a part of item l % 16, and
    // the lanes with l / 16 = l % 4 get the sum of theirs.
    auto settle = [&](int n, auto item_of) {  // item: row of the workgroup * R + column
        for (int i0 = 16 * wave; i0 < n; i0 += THREADS / 4) {
            const uint32_t item = item_of(min(i0 + (lane & 15), n - 1));
            uint4 x[4];
            hash_load_x(Kh + (first + (int)(item / R)) * a.st, x);
            const float* wc = a.W_H + ((int64_t)h * HATA_D + 32 * (lane >> 4)) * R + item % R;
            float wv[32];
#pragma unroll
            for (int s = 0; s < 32; ++s) wv[s] = wc[s * R];
            double acc = 0.0;
#pragma unroll
            for (int s = 0; s < 32; ++s) {
                const uint32_t pair = (&x[s / 8].x)[s / 2 % 4];
                acc = __builtin_amdgcn_mfma_f64_4x4x4f64((double)wv[s], (double)(s % 2 ? bf16_hi(pair) : bf16_lo(pair)), acc, 0, 0, 0);
            }
            if (lane >> 4 == (lane & 3) && i0 + (lane & 15) < n) {
                uint32_t* word = &s_code[item / 32];
                if (acc >= 0.0) atomicOr(word, 1u << (item % 32));
                else atomicAnd(word, ~(1u << (item % 32)));
            }
        }
    };
    settle(min(s_doubts, WRITE_DOUBTS), [&](int i) { return s_doubt[i]; });
    for (int k = 0; k < (s_wholes ? WRITE_MAX_ROWS / 32 : 0); ++k)
        for (uint32_t rows = s_whole[k]; rows; rows &= rows - 1) {
            const uint32_t row = 32 * k + __ffs(rows) - 1;
            settle(R, [&](int i) { return row * R + i; });
        }
    __syncthreads();
    // the code words, 16 bytes a thread where a code is as long
    if constexpr (WD >= 4) {
        for (int i = tid; i < (last - first) * (WD / 4); i += THREADS) {
            const int to = s_row[i / (WD / 4)];
            if (to >= 0) *reinterpret_cast<uint4*>(a.codes + (int64_t)to * WD + i % (WD / 4) * 4) = *reinterpret_cast<const uint4*>(&s_code[i * 4]);
        }
    } else {
        for (int i = tid; i < (last - first) * WD; i += THREADS)
            if (s_row[i / WD] >= 0) a.codes[(int64_t)s_row[i / WD] * WD + i % WD] = s_code[i];
    }
}

// Rows of a workgroup: a round of as many workgroups as are resident (two of four waves on a compute unit, one of eight), or several
// equal rounds
static int write_rows_per_wg(int n, int Hkv, int r) {
    const int64_t resident = (r <= 128 ? 2 : 1) * 256;
    const int64_t stages = (n + 63) / 64;
    int64_t rounds = 1, per;
    do per = (stages * Hkv + rounds * resident - 1) / (rounds * resident), ++rounds;
    while (per > WRITE_MAX_ROWS / 64);
    while ((stages + per - 1) / per * Hkv > (rounds - 1) * resident && per < WRITE_MAX_ROWS / 64) ++per;  // (whole stages of every head)
    return (int)per * 64;
}

hipError_t launch_write_slots(const hata_ctx* c, const void* K_new, const void* V_new, int64_t stride_t, int64_t stride_h,
                              const int32_t* slots, int n_tokens, void* K_pool, void* V_pool, uint32_t* codes, int shift, int n_pages,
                              const float* W_H, hipStream_t s) {
    const hata_config& f = c->cfg;
    const WriteSlots all = {(const uint16_t*)K_new, (const uint16_t*)V_new, slots, (uint16_t*)K_pool, (uint16_t*)V_pool, codes, W_H,
                            stride_t, stride_h, n_tokens, f.Hkv, f.r, shift, n_pages << shift};
    const int most = 65535 * WRITE_ROWS;  // rows of a launch
    for (int t0 = 0; t0 < n_tokens; t0 += most) {
        WriteSlots a = all;
        a.K_new += t0 * stride_t;
        a.V_new += t0 * stride_t;
        a.slots += t0;
        a.n = std::min(most, n_tokens - t0);
        if (codes && n_tokens > HATA_WRITE_FEW && (f.r == 32 || f.r == 64 || f.r == 128 || f.r == 256)) {
            // the weight planes prepared for exactly this weight tensor, if any
            const uint4* planes = (c->prepared_W_H == W_H && c->wplanes) ? (const uint4*)c->wplanes : nullptr;
            const int per = write_rows_per_wg(a.n, f.Hkv, f.r);
            const dim3 grid((a.n + per - 1) / per, f.Hkv);
#define HATA_LAUNCH_WRITE(R_) \
    hipLaunchKernelGGL((planes ? write_mfma_kernel<R_, true> : write_mfma_kernel<R_, false>), grid, dim3(R_ <= 128 ? 256 : 512), 0, s, a, planes, per)
            if (f.r == 32) HATA_LAUNCH_WRITE(32);
            else if (f.r == 64) HATA_LAUNCH_WRITE(64);
            else if (f.r == 128) HATA_LAUNCH_WRITE(128);
            else HATA_LAUNCH_WRITE(256);
#undef HATA_LAUNCH_WRITE
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
            if (n_tokens - t0 <= most) break;
            continue;
        }
        const int cols = f.r % 64 == 0 ? 64 : 32;
        hipLaunchKernelGGL((cols == 64 ? write_few_kernel<64> : write_few_kernel<32>),
                           dim3(codes ? f.r / cols : 1, f.Hkv, (a.n + WRITE_ROWS - 1) / WRITE_ROWS), dim3(256), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (n_tokens - t0 <= most) break;  // (t0 stays below 2^31)
    }
    return hipSuccess;
}

}  // namespace hata
