// The host's products of Newton-Schulz steps (csrc/orthogonal.hip, steps_of) on matrices of one singular value, for seeded random
// polynomials from 1e-6 to 1e4: every held number is rounded to hi + lo in fp16, as on the GPU.  None may leave fp16's range, the factors
// have to be finite numbers, and the result has to follow the polynomials.
#include "../paper_2601_02360_amd/csrc/orthogonal.hip"

#include <cstdio>
#include <random>

namespace {

bool left = false;                       // fp16's range
double held(double v) {
    const float f = (float)v;
    const _Float16 hi = (_Float16)f, lo = (_Float16)(f - (float)hi);
    if (!std::isfinite((float)hi)) left = true;
    return (double)(float)hi + (double)(float)lo;
}

double walked(const Steps& s, double value) {
    double x = held(value * s.first), square[kSquaresAtOnce] = {};
    for (const Product& f : s.of) {
        if (f.step == GRAM) {
            square[f.out] = held(x * x * f.product);
        } else if (f.step == SQUARE) {
            square[f.out] = held(square[f.p] * square[f.q] * f.product + square[f.old] * f.own + (f.other >= 0 ? square[f.other] * f.more : 0.0));
        } else {
            const double next = square[f.p] * x * f.product + x * f.own;
            if (f.step == LAST) return next;
            x = held(next);
        }
    }
    return NAN;
}

// (polynomials, singular value): the value after them, and the sum of what rounding every step's numbers to one part of their size
// would make of it.
struct Exact {
    double value, sizes;
};
Exact exact(const std::vector<double>& c, double y) {
    double sizes = 1.0, most = 1.0;
    for (size_t k = 0; k < c.size(); k += 3) {
        const double a = c[k], b = c[k + 1], d = c[k + 2], z = y * y;
        sizes = sizes * (std::fabs(a) + 3 * std::fabs(b) * z + 5 * std::fabs(d) * z * z) + std::fabs(a * y) +
                std::fabs(y) * (std::fabs(b) * z + std::fabs(d) * z * z + largest_even(b, d, most * most));
        most = largest(a, b, d, most);
        sizes += most;
        y *= a + z * (b + z * d);
    }
    return {y, sizes};
}

bool fine(const std::vector<double>& c, int steps, bool at_once, bool needed) {
    Steps s;
    if (!steps_of(c.data(), steps, at_once, s)) return !needed;
    bool ok = true;
    for (const Product& f : s.of) ok &= std::isfinite(f.product) && std::isfinite(f.own) && std::isfinite(f.more);
    for (double value : {1.0, 0.83, 0.5, 0.31, 0.1, 0.03, 1e-3}) {
        const double got = walked(s, value);
        const Exact want = exact(c, value);
        // (several steps at once lose alpha times as much, and a result below fp32's range is one)
        if (want.sizes > 1e-30) ok &= std::fabs(got - want.value) <= std::ldexp(at_once ? 4 * kMostAlpha : 1.0, -22) * want.sizes;
    }
    if (!ok || left) {
        printf("at once %d, range left %d:", at_once, left);
        for (double v : c) printf(" %g", v);
        printf("\n");
    }
    return ok && !left;
}

}  // namespace

int main() {
    // what shrinks X and lets it grow again
    for (bool at_once : {false, true}) {
        if (!fine({1e-4, 0, 0, 1e-4, 0, 0, 1e-4, 0, 0, 1e4, 0, 0, 1e4, 0, 0, 1e4, 0, 0}, 6, at_once, true)) return 1;
        if (!fine({1e-30, 0, 0, 1e4, 0, 0, 1e4, 0, 0, 1e4, 0, 0, 1e4, 0, 0}, 5, at_once, true)) return 1;
        if (!fine({1e-3, 0, 0, 0, 1e4, 0, 1e4, 0, 0}, 3, at_once, true)) return 1;
        if (!fine({0, 0, 0}, 1, at_once, true)) return 1;
    }
    std::mt19937_64 gen(1);
    auto uniform = [&](double low, double high) { return std::uniform_real_distribution<double>(low, high)(gen); };
    for (int i = 0; i < 100000; ++i) {
        const int steps = 1 + (int)(gen() % 6);
        std::vector<double> c;
        for (int k = 0; k < 3 * steps; ++k) {
            const double size = std::pow(10.0, gen() % 4 == 0 ? uniform(-6, 4) : uniform(-1, 1.5));
            c.push_back(gen() % 6 == 0 ? 0.0 : gen() % 2 ? size : -size);
        }
        if (!fine(c, steps, false, false) || !fine(c, steps, true, false)) return 1;
    }
    printf("ok\n");
    return 0;
}
