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
// 1 / (1 + exp(-x)) and what it lacks to 1, neither by a difference.  Below x = -88 the exponential is infinite and the value 0, whatever g it is multiplied with
// (held at 2^126 instead, it gave -1e36 2^-126 = -0.012 there).  What it lacks is then 0 too, not 1: it is met only as value rest.  An infinite g
// gives what its formula gives, NaN where it meets a 0.
struct Sigmoid {
    float value, rest;
};
__device__ __forceinline__ Sigmoid sigmoid(float x)
{
    const float t = fast_exp2(-1.4426950408889634f * x), s = __builtin_amdgcn_rcpf(1.f + t);
    return {s, fminf(t, 3.4028235e38f) * s};
}
template <bool SLOPE, int ACT>
__device__ __forceinline__ Act activate(float g)
{
    if (ACT == HDT_SILU) {
        const Sigmoid s = sigmoid(g);
        return {g * s.value, SLOPE ? s.value * fmaf(g, s.rest, 1.f) : 0.f};
    }
    if (ACT == HDT_GELU) {
        // Phi by erf(x) = 1 - (a1 t + .. + a5 t^5) exp(-x^2), t = 1 / (1 + p x), x >= 0, within 1.5e-7 (Hastings; Abramowitz and Stegun 7.1.26)
        const float e = fast_exp2(-0.72134752044448170f * g * g), t = __builtin_amdgcn_rcpf(fmaf(0.3275911f * 0.70710678118654752f, fabsf(g), 1.f));
        const float poly = fmaf(fmaf(fmaf(fmaf(1.061405429f, t, -1.453152027f), t, 1.421413741f), t, -0.284496736f), t, 0.254829592f);
        const float q = 0.5f * t * poly * e, cdf = g < 0.f ? q : 1.f - q;
        return {g * cdf, SLOPE ? fmaf(g * 0.3989422804014327f, e, cdf) : 0.f};
    }
    // (1 + tanh z) / 2 = sigmoid(2 z).  Beyond |g| = 15 both are what they are there, but g^2 would overflow.
    const float q = fminf(g * g, 225.f);
    const Sigmoid s = sigmoid(g * fmaf(1.5957691216057308f * 0.044715f, q, 1.5957691216057308f));
    return {g * s.value, SLOPE ? fmaf(g * s.value * s.rest, fmaf(1.5957691216057308f * 0.134145f, q, 1.5957691216057308f), s.value) : 0.f};
}
// f(activation as a constant)
template <int N>
struct Constant {
    static constexpr int value = N;
};
template <typename F>
__device__ __forceinline__ void by_act(int act, F f)
{
    if (act == HDT_SILU)
        f(Constant<HDT_SILU>());
    else if (act == HDT_GELU)
        f(Constant<HDT_GELU>());
    else
        f(Constant<HDT_GELU_TANH>());
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
