// Rotary positions of packed rows (hata_rotate), and of the rows that go into pages (the first launch of
// hata_rotate_write_slots).
#include <math.h>
#include <algorithm>
#include "hata_internal.h"
#include "hata_rotary.h"

namespace hata {

// A wave has a packed row and `per` of its heads, eight at a time: lane = (head % 8, piece of 32 bytes).  The angles of the
// row's pairs, one a lane, pass through LDS.
#define ROTATE_WAVES 4

__global__ __launch_bounds__(64 * ROTATE_WAVES) void rotate_kernel(const RotateRows a) {
    __shared__ double s_cos[ROTATE_WAVES][HATA_D / 2], s_sin[ROTATE_WAVES][HATA_D / 2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool row = (int)blockIdx.x * ROTATE_WAVES + wave < a.n;
    const int t = row ? blockIdx.x * ROTATE_WAVES + wave : a.n - 1;
    const int pairs = a.dims / 2, heads = a.heads + 2 * a.Hkv;
    if (lane < pairs) {
        double c, s;
        cos_sin((double)a.positions[t] * a.freq[lane], c, s);
        s_cos[wave][lane] = c * a.magnitude;
        s_sin[wave][lane] = (a.back ? -s : s) * a.magnitude;
    }
    __syncthreads();
    const int p = lane & 7;
    double c[8], s[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        c[i] = s_cos[wave][min(8 * p + i, pairs - 1)];
        s[i] = s_sin[wave][min(8 * p + i, pairs - 1)];
    }
    const RotaryPiece piece(p, a.dims, a.interleaved);
    const int slot = a.Hkv ? a.slots[t] : -1;
    const bool live = slot >= 0 && slot < a.rows;
    const int h_end = row ? min(heads, (int)(blockIdx.y + 1) * a.per) : 0;
    for (int h = blockIdx.y * a.per + (lane >> 3); h < h_end; h += 8) {
        const int kv = (h - a.heads) % max(a.Hkv, 1);
        const bool is_q = h < a.heads, is_k = !is_q && h < a.heads + a.Hkv;
        if (!is_q && !live) continue;
        const uint16_t* from = is_q ? a.x + t * a.st + h * a.sh : (is_k ? a.K_new : a.V_new) + t * a.kv_st + kv * a.kv_sh;
        uint16_t* to = is_q ? a.out + t * a.out_st + h * a.out_sh
                            : (is_k ? a.K : a.V) + ((((int64_t)(slot >> a.shift) * a.Hkv + kv) << a.shift) + (slot & ((1 << a.shift) - 1))) * HATA_D;
        uint4 x[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) x[i] = *reinterpret_cast<const uint4*>(from + piece.at[i]);
        if ((is_q || is_k) && 16 * p < a.dims) rotate_piece(x, c, s, a.interleaved);
#pragma unroll
        for (int i = 0; i < 2; ++i) *reinterpret_cast<uint4*>(to + piece.at[i]) = x[i];
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
        a.per = 8;
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
        const double first = std::max(floor(at(sc->high)), 0.0), last = std::min(ceil(at(sc->low)), (double)(pairs - 1));
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
