// Rotary positions of packed rows (hata_rotate), and of the rows that go into pages (the first launch of
// hata_rotate_write_slots).
#include <math.h>
#include <algorithm>
#include "hata_encode_core.h"
#include "hata_internal.h"
#include "hata_rotary.h"

namespace hata {

// A wave has a packed row and `per` of its heads, eight at a time: lane = (head % 8, piece of 32 bytes).  The angles of the
// row's pairs, one a lane, pass through LDS.  Bound by the bytes, 256 read and written a row and head: the requests of ROTATE_BATCH
// times eight heads are outstanding together.  All heads by one wave from 2048 rows on (the angles once), else eight, or a few rows would
// be as many waves: one row of 40 heads 3.4 us (the host needs 5 a call), 6001 rows of 72 heads 45 us, 4.9 TB/s, where a large copy reaches 4.8.
#define ROTATE_WAVES 4
#define ROTATE_BATCH 3

__global__ __launch_bounds__(64 * ROTATE_WAVES) void rotate_kernel(const RotateRows a) {
    __shared__ double s_cos[ROTATE_WAVES][HATA_D / 2], s_sin[ROTATE_WAVES][HATA_D / 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int t = min((int)blockIdx.x * ROTATE_WAVES + wave, a.n - 1), p = lane & 7;
    const RotaryPiece piece(p, a.dims, a.interleaved);
    const int slot = a.Hkv ? a.slots[t] : -1;
    // heads: the queries, the keys, the values; the last ones only where the row has a slot
    const int keys = a.Hkv;
    int h_end = slot >= 0 && slot < a.rows ? a.heads + 2 * keys : a.heads;
    if ((int)blockIdx.x * ROTATE_WAVES + wave >= a.n) h_end = 0;
    h_end = min(h_end, (int)(blockIdx.y + 1) * a.per);
    const uint16_t *x_row = a.x + t * a.st, *k_row = a.K_new + t * a.kv_st, *v_row = a.V_new + t * a.kv_st;
    uint16_t* out_row = a.out + t * a.out_st;
    const int64_t kv_at = ((((int64_t)(slot >> a.shift) * a.Hkv) << a.shift) + (slot & ((1 << a.shift) - 1))) * HATA_D;
    auto source = [&](int h) {
        return h < a.heads ? x_row + h * a.sh : h < a.heads + keys ? k_row + (h - a.heads) * a.kv_sh : v_row + (h - a.heads - keys) * a.kv_sh;
    };
    auto target = [&](int h) {
        return h < a.heads ? out_row + h * a.out_sh
               : h < a.heads + keys ? a.K + kv_at + ((int64_t)(h - a.heads) << a.shift) * HATA_D
                                    : a.V + kv_at + ((int64_t)(h - a.heads - keys) << a.shift) * HATA_D;
    };
    uint4 x[ROTATE_BATCH][2];
    auto load = [&](int h0) {
#pragma unroll
        for (int j = 0; j < ROTATE_BATCH; ++j)
            if (h0 + 8 * j < h_end) {
                const uint16_t* from = source(h0 + 8 * j);
#pragma unroll
                for (int i = 0; i < 2; ++i) x[j][i] = load_once(from + piece.at[i]);
            }
    };
    const int first = blockIdx.y * a.per + (lane >> 3);
    load(first);
    const int pairs = a.dims / 2;
    if (lane < pairs) {
        double c, s;
        cos_sin((double)a.positions[t] * a.freq[lane], c, s);
        s_cos[wave][lane] = c * a.magnitude;
        s_sin[wave][lane] = (a.back ? -s : s) * a.magnitude;
    }
    __syncthreads();
    double c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        c[i] = s_cos[wave][min(8 * p + i, pairs - 1)];
        s[i] = s_sin[wave][min(8 * p + i, pairs - 1)];
    }
    for (int h0 = first; h0 < h_end; h0 += 8 * ROTATE_BATCH) {
#pragma unroll
        for (int j = 0; j < ROTATE_BATCH; ++j) {
            const int h = h0 + 8 * j;
            if (h < h_end) {
                if (h < a.heads + keys && 16 * p < a.dims) rotate_piece(x[j], c, s, a.interleaved);
                uint16_t* to = target(h);
#pragma unroll
                for (int i = 0; i < 2; ++i) *reinterpret_cast<uint4*>(to + piece.at[i]) = x[j][i];
            }
        }
        load(h0 + 8 * ROTATE_BATCH);
    }
}

hipError_t launch_rotate(const RotateRows& all, hipStream_t s) {
    const int most = 1 << 20;  // rows of a launch
    const int heads = all.heads + 2 * all.Hkv;
    for (int t0 = 0; t0 < all.n;) {
        RotateRows a = all;
        a.n = std::min(most, all.n - t0);
        a.x += t0 * all.st;
        a.out += t0 * all.out_st;
        a.K_new += t0 * all.kv_st;
        a.V_new += t0 * all.kv_st;
        a.positions += t0;
        if (all.slots) a.slots += t0;
        // all heads by one wave, unless the rows are so few that the waves are
        a.per = a.n >= 2048 ? (heads + 7) / 8 * 8 : 8;
        hipLaunchKernelGGL(rotate_kernel, dim3((a.n + ROTATE_WAVES - 1) / ROTATE_WAVES, (heads + a.per - 1) / a.per), dim3(64 * ROTATE_WAVES), 0, s, a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (all.n - t0 <= most) break;
        t0 += most;
    }
    return hipSuccess;
}

// Radians a position of every pair, base^(-i / pairs), and their scalings.  (Host.)
int rotary_frequencies(int pairs, double base, const hata_rotary_scaling* sc, double* freq, float* magnitude) {
    const double two_pi = 6.28318530717958647693;
    double m = 1.0;
    for (int i = 0; i < pairs; ++i) freq[i] = pow(base, -(double)i / pairs);
    if (sc && sc->kind == HATA_ROTARY_LINEAR) {
        for (int i = 0; i < pairs; ++i) freq[i] /= sc->factor;
    } else if (sc && sc->kind == HATA_ROTARY_BASE) {
        const double b = base * pow(sc->factor, pairs > 1 ? (double)pairs / (pairs - 1) : 1.0);
        for (int i = 0; i < pairs; ++i) freq[i] = pow(b, -(double)i / pairs);
    } else if (sc && sc->kind == HATA_ROTARY_BANDS) {
        for (int i = 0; i < pairs; ++i) {
            const double turns = sc->original * freq[i] / two_pi;
            const double keep = std::min(std::max((turns - sc->low) / (sc->high - sc->low), 0.0), 1.0);
            freq[i] = freq[i] * keep + freq[i] / sc->factor * (1.0 - keep);
        }
    } else if (sc && sc->kind == HATA_ROTARY_RAMP) {
        auto at = [&](double turns) { return pairs * log(sc->original / (turns * two_pi)) / log(base); };
        const double first = std::max(floor(at(sc->high)), 0.0), last = std::min(ceil(at(sc->low)), 2.0 * pairs - 1.0);
        // (`last` may lie behind the last pair, up to dims - 1: a pair that still makes more than `low` turns is on the ramp, not at its end)
        for (int i = 0; i < pairs; ++i) {
            const double keep = 1.0 - std::min(std::max((i - first) / std::max(last - first, 1e-3), 0.0), 1.0);
            freq[i] = freq[i] * keep + freq[i] / sc->factor * (1.0 - keep);
        }
        m = sc->factor > 1.0 ? 0.1 * log(sc->factor) + 1.0 : 1.0;
    }
    *magnitude = (float)m;
    return HATA_OK;
}

}  // namespace hata
