"""Which head vectors of two sides of a rotation share memory (csrc/rope_heads.h),
compiled on its own and compared with the sets of their bytes: no GPU."""
import random
import subprocess

import pytest

from paper_2607_01817_amd import build

DRIVER = r"""
#include <cstdio>
#include "rope_heads.h"
int main() {
    long long p[2], token[2], head[2], S[2], bytes;
    int heads[2];
    while (std::scanf("%lld", &bytes) == 1) {
        hcms::HeadBlock b[2];
        for (int i = 0; i < 2; ++i) {
            if (std::scanf("%lld %lld %lld %lld %d", p + i, token + i, head + i, S + i, heads + i) != 5) return 1;
            b[i] = {static_cast<uintptr_t>(p[i]), token[i], head[i], S[i], bytes, heads[i]};
        }
        std::printf("%d\n", hcms::heads_meet(b[0], b[1]) ? 1 : 0);
    }
}
"""


@pytest.fixture(scope="module")
def meet(tmp_path_factory):
    d = tmp_path_factory.mktemp("ropeheads")
    (d / "driver.cpp").write_text(DRIVER)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", build.CSRC, str(d / "driver.cpp"), "-o",
                    str(d / "driver")], check=True)

    def ask(cases):
        text = "".join(f"{n} " + " ".join(str(v) for s in sides for v in s) + "\n" for n, *sides in cases)
        out = subprocess.run([str(d / "driver")], input=text, text=True, capture_output=True, check=True).stdout
        return [line == "1" for line in out.split()]

    return ask


def _bytes(n, p, token, head, S, heads):
    return {p + t * token + h * head + i for t in range(S) for h in range(heads) for i in range(n)}


def test_packed_sides(meet):
    """Queries, keys and values of one packed buffer of 5 tokens of 12 heads of 8 bytes:
    one after the other, and taking turns."""
    q, k, v = (96, 8, 5, 4), (96, 8, 5, 4), (96, 8, 5, 4)
    turn = (96, 24, 5, 4)
    cases = [(8, (1000, *q), (1032, *k), False), (8, (1032, *k), (1064, *v), False), (8, (1064, *v), (1000, *q), False),
             (8, (1000, *q), (1031, *k), True), (8, (1000, *q), (1024, *k), True), (8, (1000, *q), (1000, *q), True),
             (8, (1000, *turn), (1008, *turn), False), (8, (1016, *turn), (1008, *turn), False),
             (8, (1000, *turn), (1010, *turn), False), (8, (1000, *turn), (1018, *turn), True), (8, (1000, *turn), (1024, *turn), True),
             # head-major: whole sides apart, and one head shared
             (8, (1000, 8, 40, 5, 4), (1160, 8, 40, 5, 4), False), (8, (1000, 8, 40, 5, 4), (1120, 8, 40, 5, 4), True),
             # a k that starts before the last q of the token before ends
             (8, (1000, *q), (1000 + 96 + 24, *k), True), (8, (1000, *q), (1000 + 96 - 32, *k), False)]
    for *c, want in cases:
        assert bool(_bytes(c[0], *c[1]) & _bytes(c[0], *c[2])) == want, c
    assert meet([c[:-1] for c in cases]) == [c[-1] for c in cases]


def test_against_the_sets_of_bytes(meet):
    """Never False for sides that share a byte; exact where single tokens or equal token
    strides with heads between two tokens say so, but for sides of which one ends
    before the other begins to repeat."""
    rng = random.Random(5)
    cases = []
    for _ in range(4000):
        n, S = rng.randint(1, 6), rng.choice((1, 1, 2, 3, 7))
        sides = []
        token = rng.randint(0, 60)
        for _ in range(2):
            sides.append((rng.randint(100, 190), token if rng.random() < 0.8 else rng.randint(0, 60), rng.randint(0, 14), S,
                          rng.randint(1, 5)))
        cases.append((n, *sides))
    exact = 0
    for (n, a, b), got in zip(cases, meet(cases)):
        want = bool(_bytes(n, *a) & _bytes(n, *b))
        assert got or not want, (n, a, b)
        S, fits = a[3], a[1] == b[1] and all((s[4] - 1) * s[2] + n <= s[1] for s in (a, b))
        if S == 1 or (fits and abs(a[0] - b[0]) < a[1]):
            exact += 1
            assert got == want, (n, a, b)
    assert exact > 1500
