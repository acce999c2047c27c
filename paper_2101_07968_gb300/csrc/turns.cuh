// Frequencies of the rotation by position, on the host: base^(-2i / rotary) / (2 pi) turns a position, to 128 bits
// after the binary point, so that the product with any 64-bit position, modulo one turn, is good to 2^-48 of a turn.
// In integers: the same on every machine, and no compiler's contraction of floating-point operations matters.
#pragma once

#include <cmath>
#include <cstdint>

namespace dc {

using uint128 = unsigned __int128;

// m 2^e with the top bit of m set; products are cut off, 2^-127 of their value each.
struct Big {
    uint128 m;
    int e;
};
inline uint128 high_product(uint128 a, uint128 b)
{
    const uint64_t a1 = uint64_t(a >> 64), a0 = uint64_t(a), b1 = uint64_t(b >> 64), b0 = uint64_t(b);
    const uint128 low = uint128(a0) * b0, mid1 = uint128(a1) * b0, mid2 = uint128(a0) * b1;
    const uint128 carry = (low >> 64) + uint64_t(mid1) + uint64_t(mid2);
    return uint128(a1) * b1 + (mid1 >> 64) + (mid2 >> 64) + (carry >> 64);
}
inline Big times(Big a, Big b)
{
    Big p = {high_product(a.m, b.m), a.e + b.e + 128};
    if (!(p.m >> 127)) {
        p.m <<= 1;
        --p.e;
    }
    return p;
}
inline Big big_of(double x)  // x > 0
{
    int e;
    const uint64_t m = uint64_t(std::ldexp(std::frexp(x, &e), 64));
    return {uint128(m) << 64, e - 128};
}
// base^(-1 / n) for 1 <= n <= 128, base within [2^-10, 2^100]: Newton's method on base g^n = 1 from the
// double's root. Each step squares the error (n 2^-52, then 2^-85 and less, then what the products cut off).
inline Big inverse_root(double base, int n)
{
    Big g = big_of(std::pow(base, -1.0 / n));
    for (int step = 0; step < 3; ++step) {
        Big p = big_of(base), square = g;
        for (int k = n; k; k /= 2) {
            if (k & 1) p = times(p, square);
            if (k > 1) square = times(square, square);
        }
        // 1 - p in units of 2^-127; p is 1 within n 2^-51
        const uint128 at = p.e == -127 ? p.m : p.m >> 1;
        const uint128 one = uint128(1) << 127;
        const bool low = at < one;
        const uint128 by = (low ? one - at : at - one) / unsigned(n), change = high_product(g.m, by) << 1;
        const uint128 was = g.m;
        g.m = low ? g.m + change : g.m - change;
        if (low ? g.m < was : !(g.m >> 127)) {  // past a power of two
            g.m = low ? (g.m >> 1) | one : g.m << 1;
            g.e += low ? 1 : -1;
        }
    }
    return g;
}
// Frequencies of pairs 0 .. half - 1, the fraction's upper and lower 64 bits; whole turns are left out.
inline void rotary_turns(double base, int half, uint64_t *upper, uint64_t *lower)
{
    if (half == 0) return;
    const Big g = inverse_root(base, half);
    // 1 / (2 pi) = 0.a2f9836e.. 2^-2
    Big f = {uint128(0xa2f9836e4e441529ull) << 64 | 0xfc2757d1f534ddc0ull, -130};
    for (int i = 0; i < half; ++i) {
        const int up = f.e + 128;
        const uint128 part = up >= 128 || up <= -128 ? uint128(0) : up >= 0 ? f.m << up : f.m >> -up;
        upper[i] = uint64_t(part >> 64);
        lower[i] = uint64_t(part);
        f = times(f, g);
    }
}

}  // namespace dc
