// How far an orthogonalised matrix' singular values may go (ortho_reach, ortho_units of csrc/fsa_block.h): the estimate against the polynomials
// at many points, and planes that hold it.
#include "../../paper_2511_13645_amd/csrc/fsa_block.h"

#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>

using namespace fsa;

#define CHECK(x) do { if (!(x)) { std::printf("%s: %g %g %g from %g\n", #x, abc[0], abc[1], abc[2], reach); std::exit(1); } } while (0)

int main() {
    std::mt19937_64 rng(7);
    auto uniform = [&](double lo, double hi) { return lo + (hi - lo) * (double)(rng() >> 11) * 0x1p-53; };
    for (int round = 0; round < 20000; ++round) {
        const double reach = std::exp2(uniform(-3.0, 4.0)), size = std::exp2(uniform(-6.0, 6.0));
        float abc[3] = {(float)uniform(-size, size), (float)uniform(-size, size), (float)uniform(-size, size)};
        for (float& x : abc) if (rng() % 6 == 0) x = rng() % 2 ? 0.0f : x * 1e-30f;
        const OrthoReach r = ortho_reach(abc, reach);
        double poly = 0.0, next = 0.0;
        constexpr int kPoints = 400;
        for (int i = 0; i <= kPoints; ++i) {
            const double s = reach * i / kPoints, t = s * s, p = abc[1] * t + abc[2] * t * t;
            poly = std::fmax(poly, std::fabs(p));
            next = std::fmax(next, std::fabs(s * (abc[0] + p)));
        }
        CHECK(poly <= r.poly * (1 + 1e-12) + 1e-300 && next <= r.next * (1 + 1e-12) + 1e-300);
        // no more than the points miss of a smooth curve between them: an eighth of a step's square of its bend
        const double step = reach / kPoints, bend = 2 * std::fabs(abc[1]) + 12 * std::fabs(abc[2]) * reach * reach;
        CHECK(r.poly <= poly * (1 + 1e-12) + step * step * bend && r.next <= next * (1 + 1e-12) + step * step * reach * (6 * std::fabs(abc[1]) + 20 * std::fabs(abc[2]) * reach * reach));
        for (int most : {kUnitX, kUnitP}) {
            const int unit = ortho_unit(r.poly, most);
            CHECK(unit <= most && std::ldexp(r.poly, unit) <= kMostHeld && (unit == most || std::ldexp(r.poly, unit + 1) > kMostHeld));
        }
    }
    double reach = 1.0;
    {
        // singular values that stay small have the usual units; larger ones give way
        float abc[12] = {3.4445f, -4.7750f, 2.0315f, 3.4445f, -4.7750f, 2.0315f, 16.0f, 16.0f, 16.0f, 1.0f, 0.0f, 0.0f};
        OrthoUnits u[4];
        CHECK(ortho_units(abc, 4, 16.0, u));
        for (int i = 0; i < 2; ++i) CHECK(u[i].x == kUnitX && u[i].a == kUnitA && u[i].p == kUnitP);
        CHECK(u[3].x < kUnitX && u[3].a < u[3].x);
    }
    {
        // coefficients beyond 16: taken where singular values of one and below stay below 8
        float abc[6] = {8.0f, -23.0f, 16.5f, 1.766f, -0.644f, 0.072f};
        OrthoUnits u[2];
        CHECK(ortho_units(abc, 2, 16.0, u));
        abc[1] = 23.0f;
        CHECK(!ortho_units(abc, 2, 16.0, u));
        abc[0] = 0.0f; abc[1] = 17.0f; abc[2] = 0.0f;
        CHECK(!ortho_units(abc, 1, 16.0, u));
        abc[0] = 1025.0f; abc[1] = -1025.0f;
        CHECK(!ortho_units(abc, 1, 16.0, u));
        abc[0] = NAN; abc[1] = 0.0f;
        CHECK(!ortho_units(abc, 1, 16.0, u));
        // and up to 16 whatever becomes of them
        for (float& x : abc) x = 16.0f;
        CHECK(ortho_units(abc, 2, 16.0, u));
        float many[96];
        OrthoUnits all[32];
        for (float& x : many) x = 16.0f;
        CHECK(ortho_units(many, 32, 16.0, all) && all[31].x == kLeastUnit && all[31].p == kLeastUnit);
    }
    std::puts("ok");
}
