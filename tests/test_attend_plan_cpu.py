"""The attention operators' host-side plan (csrc/iso_grad_plan.cpp): pieces, the workspace that they take and the launches."""
import random

import pytest

from tests.grad_plan_program import program

# of every line's tokens_q tokens_k sequences heads heads_kv dim: the plan of both calls
PLAN = r"""int main() {
  long long q, k, s;
  int h, kv, d;
  while (scanf("%lld %lld %lld %d %d %d", &q, &k, &s, &h, &kv, &d) == 6) {
    iso_attn a{};
    a.tokens_q = q, a.tokens_k = k, a.sequences = s, a.heads = h, a.heads_kv = kv, a.dim = d;
    const AttendPlan F = plan_attend(a, false), B = plan_attend(a, true);
    const long long list = q * (h / kv);
    printf("%d %d %d %d %d %d %zu %zu %zu %zu %zu %u %u %d\n", F.rows.most, F.rows.keys, B.rows.most, B.rows.keys, B.keys.most, B.keys.keys,
           F.part, F.total, B.part, B.key_part, B.total, attend_items(list, k, s, B.rows), attend_items(k, list, s, B.keys), (int)kPartLd);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    import subprocess
    path = tmp_path_factory.mktemp("attend_plan")
    program(path, PLAN)

    def run(cases):
        text = "".join(" ".join(map(str, c)) + "\n" for c in cases)
        out = subprocess.run([str(path / "t")], input=text, check=True, capture_output=True, text=True).stdout
        return [[int(x) for x in line.split()] for line in out.splitlines()]
    return run


def cases():
    rng = random.Random(5)
    yield (457, 400000, 1, 7, 1, 8)      # a tile is shared out to most pieces, and is nearly two
    yield (1, 1 << 20, 1, 28, 4, 128)
    yield (1, 0, 1, 4, 2, 64)
    for _ in range(4000):
        kv = rng.choice([1, 2, 3, 4, 8, 12])
        heads = kv * rng.choice([1, 2, 7, 8, 64])
        q = int(2 ** rng.uniform(0, 22)) * 4 // heads + 1
        k = int(2 ** rng.uniform(0, 25)) // kv + 1
        yield (q, k, int(2 ** rng.uniform(0, 8)), heads, kv, 64)
    for rows in range(60, 3400, 1):      # around every step of the number of tiles
        yield (rows, 600000, 1, 1, 1, 64)
        yield (600000, rows, 1, 1, 1, 64)


def test_pieces_fit_the_workspace(plan):
    todo = list(cases())
    for c, p in zip(todo, plan(todo)):
        q, k, s, h, kv, d = c
        f_most, _, b_most, _, k_most, _, f_part, f_total, b_part, key_part, total, _, _, ld = p
        assert f_most >= 1 and k_most >= 1 and f_most == b_most, c
        assert f_most == 1 or f_total - f_part >= 4 * ld * f_most * q * h, c
        assert b_most == 1 or key_part - b_part >= 4 * ld * b_most * q * h, c
        assert k_most == 1 or total - key_part >= 8 * ld * k_most * k * kv, c
        assert b_part >= 256 + 4 * (2 * q * h + 64), c


def test_workspace_does_not_fall_with_tokens_or_sequences(plan):
    rng = random.Random(6)
    small, large = [], []
    for _ in range(4000):
        kv, g = rng.choice([1, 2, 4]), rng.choice([1, 2, 7])
        q, k, s = int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 20)), int(2 ** rng.uniform(0, 7))
        small.append((q, k, s, kv * g, kv, 64))
        large.append((q + rng.choice([0, 1, 127, q]), k + rng.choice([0, 1, 255, k]), s + rng.choice([0, 1, s]), kv * g, kv, 64))
    for c, a, b in zip(small, plan(small), plan(large)):
        assert a[7] <= b[7] and a[10] <= b[10], c


def test_launches_hold_every_sequences_items(plan):
    """Tiles of 128 rows (keys), pieces of at least `keys` keys (rows), at most `most`: a launch's items are an upper bound."""
    rng = random.Random(7)
    todo, lens = [], []
    for _ in range(2000):
        s = rng.choice([1, 2, 5, 64, 200])
        top = 2 ** rng.uniform(0, 14 if s < 64 else 9)
        nq = [int(rng.uniform(0, top)) for _ in range(s)]
        nk = [int(rng.uniform(0, top)) * rng.choice([0, 1, 1, 20]) for _ in range(s)]
        kv, g = rng.choice([1, 2, 4]), rng.choice([1, 2, 7])
        todo.append((sum(nq), sum(nk), s, kv * g, kv, 64))
        lens.append((nq, nk, g))
    for c, p, (nq, nk, g) in zip(todo, plan(todo), lens):
        rows_most, rows_keys, k_most, k_keys = p[2], p[3], p[4], p[5]
        pieces = lambda n, most, each: min(most, max(1, -(-n // each)))  # noqa: E731
        assert p[11] >= sum(-(-n * g // 128) * pieces(m, rows_most, rows_keys) for n, m in zip(nq, nk)), c
        assert p[12] >= sum(-(-m // 128) * pieces(n * g, k_most, k_keys) for n, m in zip(nq, nk)), c
