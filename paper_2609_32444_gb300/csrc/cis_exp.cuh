// cis_exp.cuh -- exponentials right to 2^-42, as pairs of fp32 numbers: the masses in whole
// numbers of the sampler and the lists, and the sum of a list's probabilities, which 1 is nearly.
#pragma once

#include "cis_common.cuh"

namespace cis {
namespace {

// 2^{i/32} as fp32 pairs.
__device__ const float2 kExp2Table[32] = {
    {1.0f, 0.0f}, {0x1.059b0ep0f, -0x1.9d4f52p-25f},
    {0x1.0b5586p0f, 0x1.9f3122p-25f}, {0x1.11301ep0f, -0x1.fdb496p-25f},
    {0x1.172b84p0f, -0x1.c15742p-27f}, {0x1.1d4874p0f, -0x1.d2e8cap-25f},
    {0x1.2387a6p0f, 0x1.ceac48p-25f}, {0x1.29e9ep0f, -0x1.5c0424p-25f},
    {0x1.306fep0f, 0x1.4636e2p-25f}, {0x1.371a74p0f, -0x1.18aac6p-25f},
    {0x1.3dea64p0f, 0x1.824684p-25f}, {0x1.44e086p0f, 0x1.8624b4p-30f},
    {0x1.4bfdaep0f, -0x1.593abcp-25f}, {0x1.5342b6p0f, -0x1.2c561p-25f},
    {0x1.5ab07ep0f, -0x1.5bd5ecp-27f}, {0x1.6247ecp0f, -0x1.f8b55p-25f},
    {0x1.6a09e6p0f, 0x1.9fcef4p-26f}, {0x1.71f75ep0f, 0x1.1d8beep-25f},
    {0x1.7a1148p0f, -0x1.829fdp-25f}, {0x1.82589ap0f, -0x1.accc7cp-26f},
    {0x1.8ace54p0f, 0x1.15506ep-27f}, {0x1.93737cp0f, -0x1.e64744p-25f},
    {0x1.9c4918p0f, 0x1.51f848p-27f}, {0x1.a5503cp0f, -0x1.b83b54p-25f},
    {0x1.ae89fap0f, -0x1.a94b14p-26f}, {0x1.b7f77p0f, -0x1.a09438p-25f},
    {0x1.c199bep0f, -0x1.3d56b2p-27f}, {0x1.cb720ep0f, -0x1.8837ccp-27f},
    {0x1.d5818ep0f, -0x1.822dbcp-27f}, {0x1.dfc974p0f, -0x1.908c94p-25f},
    {0x1.ea4afap0f, 0x1.52486cp-27f}, {0x1.f50766p0f, -0x1.246ebp-26f}};

// a + b = s + e exactly, for finite numbers; ordered: |a| >= |b|.
__device__ __forceinline__ float sum_pair(float a, float b, float &e)
{
    const float s = __fadd_rn(a, b), v = __fsub_rn(s, a);
    e = __fadd_rn(__fsub_rn(a, __fsub_rn(s, v)), __fsub_rn(b, v));
    return s;
}
__device__ __forceinline__ float sum_ordered(float a, float b, float &e)
{
    const float s = __fadd_rn(a, b);
    e = __fsub_rn(b, __fsub_rn(s, a));
    return s;
}
// e^{x + x_lo} = (s + lo) 2^{n >> 5} for |x| < 31, right to 2^-42, by a table of 2^{i/32} and a
// short series (the table-driven method of P. T. P. Tang, ACM TOMS 15, 1989): x is reduced to
// n ln2/32 + r, |r| <= 0.011, with ln2/32 in three parts (n has 11 bits and the first part 12, so
// that the first product is exact), e^r is its Taylor series with the terms up to r^2/2 kept as a
// pair, and 2^{n/32} comes from the table.  s is a multiple of 2^-24 below 2.2.
__device__ __forceinline__ float exp_parts(float x, float x_lo, float &lo, int &ni)
{
    const float n = rintf(x * (32.0f * kLog2e));
    const float t0 = fmaf(n, -0x1.62ep-6f, x);
    float e1, e2, e3;
    const float p1 = n * -0x1.0bfbe8p-20f, p1e = fmaf(n, -0x1.0bfbe8p-20f, -p1);
    const float r = sum_pair(t0, p1, e1);
    const float rl = e1 + (p1e + fmaf(n, -0x1.cf79acp-45f, x_lo));
    float q = fmaf(1.0f / 120.0f, r, 1.0f / 24.0f);
    q = fmaf(q, r, 1.0f / 6.0f);
    const float h = 0.5f * r, s2 = h * r, s2e = fmaf(h, r, -s2);
    const float w = sum_ordered(r, s2, e2);  // e^{r + rl} - 1 = w + wl
    const float wl = e2 + (s2e + fmaf(q * r, r * r, fmaf(rl, w, rl)));
    ni = __float2int_rn(n);
    const float2 T = __ldg(&kExp2Table[ni & 31]);
    const float p = T.x * w, pe = fmaf(T.x, w, -p);
    const float s = sum_ordered(T.x, p, e3);
    lo = e3 + (pe + (T.y + fmaf(T.x, wl, T.y * w)));
    return s;
}

}  // namespace
}  // namespace cis
