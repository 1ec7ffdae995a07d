// Gated feed-forward block, shared by its kernels:
//
//   G = X Wg^T, U = X Wu^T, H = act(G) o U, Y = H Wd^T                                  X [rows][width], Wg, Wu [inner][width], Wd [width][inner]
//   dH = dY Wd, dG = dH o Pg, dU = dH o Pu, dX = dG Wg + dU Wu, dWg = dG^T X, dWu = dU^T X, dWd = dY^T H
//
// Pg = U o act'(G) and Pu = act(G) are H's derivatives by G and U.  The forward, which has G and U in fp32, keeps these for the backward and not
// G and U: as many bytes, the activation is evaluated once, and each gradient has one rounding of what was kept (of G and U it had two and more:
// dWg, dWu, dX 0.0030 of their norm from 64-bit values, with Pg and Pu 0.0028; results rounded once are 0.0017 off).
//
// Products are C[m][n] = sum over k of A(m, k) B(n, k), of operands whose k is consecutive in memory ("fast": [m][k]) or not ("slow": [k][m]):
//   GATE    A = X fast, B = Wg and Wu fast; both sums of a pair (m, n) come together, and Pg, Pu, H leave     (forward)
//   DGATE   A = dY fast, B = Wd slow: dH, which is not stored: dG and dU leave                                  (backward)
//   STORE   A = H fast, B = Wd fast: Y;  A = dG then dU fast, B = Wg then Wu slow: dX, k going through both;  A = dG, dU or dY slow, B = X, X
//           or H slow: the weights' gradients, k going over the rows
#pragma once

#include "hdt_internal.h"
#include "hdt_mfma.h"

namespace hdt_ffn {

enum { GATE, STORE, DGATE };

// act(g) and its derivative
struct Act {
    float value, slope;
};
// 1 / (1 + exp(-x)) and what it lacks to 1, neither by a difference.  (The exponent is bounded: an infinite exponential times zero.)
struct Sigmoid {
    float value, rest;
};
__device__ __forceinline__ Sigmoid sigmoid(float x)
{
    const float t = fast_exp2(fminf(-1.4426950408889634f * x, 126.f)), s = 1.f / (1.f + t);
    return {s, t * s};
}
template <bool SLOPE>
__device__ __forceinline__ Act activate(float g, int act)
{
    if (act == HDT_SILU) {
        const Sigmoid s = sigmoid(g);
        return {g * s.value, SLOPE ? s.value * fmaf(g, s.rest, 1.f) : 0.f};
    }
    if (act == HDT_GELU) {
        const float cdf = 0.5f * (1.f + erff(g * 0.70710678118654752f));
        return {g * cdf, SLOPE ? fmaf(g * 0.3989422804014327f, fast_exp2(-0.72134752044448170f * g * g), cdf) : 0.f};
    }
    // (1 + tanh z) / 2 = sigmoid(2 z); beyond 15 the derivative is 0 or 1, and its factors overflow
    const float q = g * g;
    const Sigmoid s = sigmoid(1.5957691216057308f * g * fmaf(0.044715f, q, 1.f));
    float slope = 0.f;
    if (SLOPE) {
        const float inner = fmaf(g * s.value * s.rest, 1.5957691216057308f * fmaf(0.134145f, q, 1.f), s.value);
        slope = g < -15.f ? 0.f : g > 15.f ? 1.f : inner;
    }
    return {g * s.value, slope};
}

struct Product {
    const void *a[2], *b[2];     // GATE: b of G and U; STORE: the two ranges of k; else the first
    int64_t lda, ldb;            // elements from row to row
    int m, n, k;                 // k: of one range
    int ranges;                  // of k: 1 or 2
    void *out[3];                // GATE: Pg, Pu (both may be NULL), H; STORE: C; DGATE: dG, dU
    const void *by_gate, *by_up; // DGATE: Pg, Pu
    int64_t ldo;                 // of out, by_gate, by_up
    int act;
};

}  // namespace hdt_ffn
