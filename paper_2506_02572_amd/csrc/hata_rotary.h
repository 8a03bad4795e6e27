// Rotary positions: pairs of channels turned by an angle that grows with the row's position,
//   y_a = m (x_a cos t - x_b sin t),  y_b = m (x_a sin t + x_b cos t),  t = position freq_i,
// evaluated in fp64 and rounded to bf16 once, so that a row has one set of bits whichever call rotates it (its key code is
// taken from those bits).  fp64 runs at the rate of fp32 here, and an angle is shared by all heads of a row.
#pragma once
#include "hata_device.h"

namespace hata {

// cos and sin of t, |t| up to 2^31 and beyond: t less the nearest multiple of pi / 2, of which 106 bits are taken (Cody and Waite), and the
// Taylor sums there, whose first terms left out are below 2^-58 of the sums
__device__ __forceinline__ void cos_sin(double t, double& c, double& s) {
    const double k = rint(t * 0.63661977236758134308);
    double r = fma(-k, 1.57079632679489655800, t);
    r = fma(-k, 6.12323399573676603587e-17, r);
    const double z = r * r;
    double ps = 1.0 / 355687428096000.0;  // 17!
    ps = fma(ps, z, -1.0 / 1307674368000.0);
    ps = fma(ps, z, 1.0 / 6227020800.0);
    ps = fma(ps, z, -1.0 / 39916800.0);
    ps = fma(ps, z, 1.0 / 362880.0);
    ps = fma(ps, z, -1.0 / 5040.0);
    ps = fma(ps, z, 1.0 / 120.0);
    ps = fma(ps, z, -1.0 / 6.0);
    const double sine = fma(ps * z, r, r);
    double pc = -1.0 / 6402373705728000.0;  // 18!
    pc = fma(pc, z, 1.0 / 20922789888000.0);
    pc = fma(pc, z, -1.0 / 87178291200.0);
    pc = fma(pc, z, 1.0 / 479001600.0);
    pc = fma(pc, z, -1.0 / 3628800.0);
    pc = fma(pc, z, 1.0 / 40320.0);
    pc = fma(pc, z, -1.0 / 720.0);
    pc = fma(pc, z, 1.0 / 24.0);
    pc = fma(pc, z, -0.5);
    const double cosine = fma(pc, z, 1.0);
    const int quarter = (int)(k - 4.0 * floor(0.25 * k));  // 0 .. 3
    const double x = quarter & 1 ? sine : cosine, y = quarter & 1 ? cosine : sine;
    c = quarter == 1 || quarter == 2 ? -x : x;
    s = quarter >= 2 ? -y : y;
}

// Two fp64 values -> two bf16, each rounded once: where the fp32 in between lies half-way between two bf16 it is moved off that,
// to the side of the value
__device__ __forceinline__ uint32_t off_half(double d) {
    uint32_t u = __float_as_uint((float)d);
    if ((u & 0xffffu) == 0x8000u) {
        const double e = fabs(d) - fabs((double)__uint_as_float(u));
        u += e > 0.0 ? 1u : e < 0.0 ? ~0u : 0u;
    }
    return u;
}
__device__ __forceinline__ uint32_t bf16_pair(double lo, double hi) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    f32x2 f;
    f[0] = __uint_as_float(off_half(lo));
    f[1] = __uint_as_float(off_half(hi));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

struct RotaryArgs {
    const double* freq;
    const int32_t* positions;
    double magnitude;
    int dims, interleaved;
};

// A row goes in eight pieces of 32 bytes.  Piece p < dims / 16 holds pairs 8 p .. 8 p + 7, as two 16-byte parts: with halves the first
// channels of those pairs and the second ones, with neighbours one behind the other.  The other pieces hold channels 16 p .. 16 p + 15.
struct RotaryPiece {
    int at[2];  // first channel of each part
    __device__ __forceinline__ RotaryPiece(int p, int dims, bool interleaved) {
        const bool halves = !interleaved && 16 * p < dims;
        at[0] = halves ? 8 * p : 16 * p;
        at[1] = halves ? dims / 2 + 8 * p : 16 * p + 8;
    }
};

// c, s: of the piece's eight pairs
__device__ __forceinline__ void rotate_piece(uint4 (&x)[2], const double (&c)[8], const double (&s)[8], bool interleaved) {
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            uint32_t& v = i < 4 ? (&x[0].x)[i] : (&x[1].x)[i - 4];
            const double a = bf16_lo(v), b = bf16_hi(v);
            v = bf16_pair(fma(a, c[i], -(b * s[i])), fma(a, s[i], b * c[i]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t &v = (&x[0].x)[i], &w2 = (&x[1].x)[i];
            const double a0 = bf16_lo(v), a1 = bf16_hi(v), b0 = bf16_lo(w2), b1 = bf16_hi(w2);
            v = bf16_pair(fma(a0, c[2 * i], -(b0 * s[2 * i])), fma(a1, c[2 * i + 1], -(b1 * s[2 * i + 1])));
            w2 = bf16_pair(fma(a0, s[2 * i], b0 * c[2 * i]), fma(a1, s[2 * i + 1], b1 * c[2 * i + 1]));
        }
    }
}

// Angles of up to 16 rows in LDS, four pairs a thread of 256
struct RotaryTable {
    double cos[16][HATA_D / 2], sin[16][HATA_D / 2];
    __device__ __forceinline__ void fill(const RotaryArgs& a, int t0, int rows) {
        const int v = threadIdx.x >> 4, pairs = a.dims / 2;
        const double position = a.positions[t0 + min(v, rows - 1)];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = (threadIdx.x & 15) + 16 * i;
            double c, s;
            cos_sin(position * a.freq[min(p, pairs - 1)], c, s);
            cos[v][p] = c * a.magnitude;
            sin[v][p] = s * a.magnitude;
        }
    }
    // piece p of row v
    __device__ __forceinline__ void rotate(const RotaryArgs& a, uint4 (&x)[2], int v, int p) const {
        if (16 * p >= a.dims) return;
        double c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c[i] = cos[v][8 * p + i];
            s[i] = sin[v][8 * p + i];
        }
        rotate_piece(x, c, s, a.interleaved);
    }
};

}  // namespace hata
