// Attention of drafted tokens on block tables (hata_dense_tree_paged), and the rows of the accepted ones (hata_keep_rows).
#include <algorithm>
#include "hata_attn_core.h"
#include "hata_device.h"
#include "hata_internal.h"

namespace hata {

// Row n of sequence b in the pools: the row of head h of its page is row_of(n) * 1 (in rows of HATA_D values)
__device__ __forceinline__ int pool_row(const PageView& pv, int b, int n, int h, int Hkv) {
    const int page = clampi(pv.table[(int64_t)b * pv.max_blocks + (n >> pv.shift)], 0, pv.n_pages - 1);
    return ((page * Hkv + h) << pv.shift) + (n & ((1 << pv.shift) - 1));
}

// A workgroup has a query head of a token; its waves take every fourth row that the token sees, a lane two channels.
__global__ __launch_bounds__(256) void tree_kernel(const TreeArgs a) {
    __shared__ float s_m[4], s_l[4], s_acc[4][HATA_D];
    const int t = blockIdx.x, hq = blockIdx.y, h = hq / a.G, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int b = 0, c = a.B;  // the last sequence that begins at t or before
    while (c > 1) {
        const int m = c / 2;
        if (a.token_start[b + m] <= t) { b += m; c -= m; }
        else c = m;
    }
    const int t0 = clampi(a.token_start[b], 0, a.n_tokens), t1 = clampi(a.token_start[b + 1], 0, a.n_tokens), i = t - t0;
    if (t < t0 || t >= t1 || i >= a.max_draft) return;
    const int L = clampi(a.seq_len[b], 0, a.L_cap), base = clampi(a.base[b], 0, L), end = min(L, base + min(t1 - t0, a.max_draft));
    const uint32_t* seen = a.mask ? a.mask + (int64_t)t * a.words : nullptr;
    const int64_t o = ((int64_t)t * a.Hq + hq) * HATA_D;
    const uint32_t q = reinterpret_cast<const uint32_t*>(a.q + o)[lane];
    float m = HATA_NEG_INF, l = 0.f, x = 0.f, y = 0.f;
    for (int n = wave; n < end; n += 4) {
        const int j = n - base;
        if (j >= 0 && !(seen ? seen[j >> 5] >> (j & 31) & 1 : j <= i)) continue;
        const int64_t row = (int64_t)pool_row(a.pv, b, n, h, a.Hkv) * HATA_D;
        const uint32_t k = reinterpret_cast<const uint32_t*>(a.K + row)[lane], v = reinterpret_cast<const uint32_t*>(a.V + row)[lane];
        const float score = wave_sum64(dot2_bf16(q, k, 0.f)) * a.scale_log2, top = fmaxf(m, score);
        const float sub = top == HATA_NEG_INF ? 0.f : top, f = fast_exp2(m - sub), p = fast_exp2(score - sub);
        l = fmaf(l, f, p);
        x = fmaf(x, f, p * bf16_lo(v));
        y = fmaf(y, f, p * bf16_hi(v));
        m = top;
    }
    if (lane == 0) { s_m[wave] = m; s_l[wave] = l; }
    s_acc[wave][2 * lane] = x;
    s_acc[wave][2 * lane + 1] = y;
    __syncthreads();
    if (threadIdx.x >= HATA_D) return;
    const float top = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3])), sub = top == HATA_NEG_INF ? 0.f : top;
    float sum = 0.f, acc = 0.f;
    for (int w = 0; w < 4; ++w) {
        const float f = fast_exp2(s_m[w] - sub);
        sum = fmaf(f, s_l[w], sum);
        acc = fmaf(f, s_acc[w][threadIdx.x], acc);
    }
    const float r = sum == 0.f && top == HATA_NEG_INF ? 0.f : acc / sum;
    a.out[o + threadIdx.x] = (uint16_t)f32_to_bf16(r);
    if (a.out_f32) a.out_f32[o + threadIdx.x] = r;
}

hipError_t launch_tree(const hata_ctx*, const TreeArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(tree_kernel, dim3(a.n_tokens, a.Hq), dim3(256), 0, s, a);
    return hipGetLastError();
}

size_t tree_scratch_bytes(int, int, int, int, int) { return 256; }

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
