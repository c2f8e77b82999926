"""Host-side plans of the gradient operators, checked on the CPU: the regions of a workspace lie apart and inside it, every
tile, copy and workgroup is accounted for, tables hold what a launch takes."""
import random

import pytest

from tests.grad_plan_program import WEIGHT_GRAD, program, schedule

BASE = 1 << 20


def layer_list(rng, n, kind):
    out = []
    for j in range(n):
        t = rng.choice([0, 1, 31, 32, 33, 700, 5000]) if kind != "large" else rng.choice([1, 8192, 65536])
        o, i = (rng.randint(1, 3000) for _ in range(2)) if kind != "large" else (rng.randint(9000, 19000) for _ in range(2))
        share = j + 1
        if kind == "shared" and out and rng.random() < 0.6:
            t, _, i, _, share = rng.choice(out)
        out.append((t, o, i, o + rng.choice([0, 0, 1, 8 - o % 8]), share))
    return out


@pytest.mark.parametrize("dt", [0, 1])
@pytest.mark.parametrize("kind", ["apart", "shared", "large"])
def test_weight_gradient_tables(tmp_path, dt, kind):
    run = program(tmp_path, WEIGHT_GRAD)
    rng = random.Random(f"{dt} {kind}")
    for n in (1, 2, 7, 15, 16):
        for accumulate in (False, True):
            layers = layer_list(rng, n, kind)
            p = schedule(run, layers, dt, accumulate, BASE)
            live = [l for l in layers if not (accumulate and l[0] == 0)]
            assert len(p.layers) == len(live) and p.tile in (128, 256)
            # tiles: one after another, as many as the matrices take; longest sums first
            at, last = 0, 1 << 40
            for y, x, g, y_ld, x_ld, y_bytes, x_bytes, rows, cols, across, down, steps, parts, tile0 in p.layers:
                t, o, i, ld, share = layers[g - 1]
                assert (rows, cols) == (o, i) and tile0 == at and steps == -(-t // 32) <= last
                assert across == -(-i // p.tile) and down == -(-o // p.tile) and parts == (3 if dt == 0 else 1)
                at, last = at + across * down, steps
            assert at == p.tiles
            units = 256 if p.tile == 256 else 512
            rest = p.tiles - p.whole
            if rest:
                assert p.whole % units == 0 and p.split > 1 and rest * p.split <= units
            else:
                assert p.split == 1
            # copies: their workgroups follow each other, their places lie apart and inside the workspace
            spans, block = [], 0
            for dst, rows, ld, part, cols, per_row, block0, is_x in p.prep:
                assert block0 == block and per_row == (-(-cols // 32) * 4 if is_x else -(-cols // 8))
                held = rows if is_x else part
                assert is_x or part == -(-rows // 32) * 32
                block += -(-held * per_row // 256)
                spans.append((dst, dst + 16 * per_row * held * (1 if is_x else p.layers[0][12])))
            assert block == p.blocks and len(p.prep) == p.preps
            if rest:
                spans.append((p.part, p.part + 4 * p.tile * p.tile * rest * p.split))
            spans.sort()
            assert all(a % 256 == 0 for a, _ in spans)
            assert not spans or spans[0][0] >= BASE + 256 and spans[-1][1] <= BASE + p.total <= BASE + p.need
            assert all(a[1] <= b[0] for a, b in zip(spans, spans[1:]))
            # operands: bf16 rows in place where they are aligned, else a copy; layers of one checkpoint share its copy
            shared = {}
            for y, x, g, y_ld, x_ld, y_bytes, x_bytes, *_ in p.layers:
                t, o, i, ld, share = layers[g - 1]
                if t == 0:
                    continue
                assert x_ld == 64 * -(-i // 32) and x_bytes == t * x_ld and x in [s for s, _ in spans]
                assert shared.setdefault((share, t, i), x) == x
                if dt == 1 and ld % 8 == 0:
                    assert y == g << 40 and y_ld == 2 * ld and 0 <= y_bytes - 2 * ((t - 1) * ld + o) < 16 and y_bytes % 16 == 0
                else:
                    assert y in [s for s, _ in spans] and y_ld == 16 * -(-o // 8)
                    assert y_bytes == (3 if dt == 0 else 1) * -(-t // 32) * 32 * y_ld
            assert len(set(shared.values())) == len(shared)


TABLES = r"""struct Arg { int64_t rows; uint32_t cols, per_row; };
struct Table { Arg t[kTable]; uint32_t block0[kTable + 1]; int n; };
int main(int n, char** v) {
  std::vector<Arg> a;
  for (int j = 3; j + 1 < n; j += 2) a.push_back(Arg{atoll(v[j]), (uint32_t)atoll(v[j + 1]), (uint32_t)(ckpt_ld(atoll(v[j + 1])) / 8)});
  for_tables<Table>(a.data(), (int)a.size(), atoi(v[1]), atoi(v[2]), [](const Arg& x) { return x; },
                    [](const Table& T, unsigned grid, int64_t bytes) {
    printf("%u %lld", grid, (long long)bytes);
    for (int j = 0; j < T.n; ++j) printf(" %lld %u %u", (long long)T.t[j].rows, T.t[j].cols, T.block0[j]);
    printf("\n");
  });
}"""


@pytest.mark.parametrize("items", [1, 2])
def test_checkpoint_tables(tmp_path, items):
    run = program(tmp_path, TABLES)
    rng = random.Random(items)
    for n in (0, 1, 16, 17, 40):
        for large in (False, True):
            shapes = [(rng.choice([0, 1, 7, 4096]), rng.choice([0, 1, 33, 18944])) if not large or rng.random() < 0.5 else
                      (rng.randint(1 << 18, 1 << 20), rng.randint(4000, 16000)) for _ in range(n)]
            done = []
            for line in run(items, 16, *[w for s in shapes for w in s]):
                grid, nbytes, *rest = map(int, line)
                table = [tuple(rest[j:j + 3]) for j in range(0, len(rest), 3)]
                assert 1 <= len(table) <= 16
                block = total = 0
                for rows, cols, block0 in table:
                    groups = rows * (-(-cols // 32) * 4)
                    assert block0 == block
                    block += -(-groups // (256 * items))
                    total += groups * 16
                assert grid == block and nbytes == total and (grid <= 1 << 22 or len(table) == 1) and grid < 1 << 24
                done += [(rows, cols) for rows, cols, _ in table]
            assert done == [s for s in shapes if s[0] and s[1]]


EMBED = r"""int main(int n, char** v) {
  const EmbedPlan P = embed_plan(atoll(v[1]), atoll(v[2]), atoll(v[3]));
  printf("%lld %lld %lld %zu", (long long)P.tiles, (long long)P.tile, (long long)P.most_runs, P.total);
  for (size_t o : {P.bad, P.hist, P.bucket0, P.pairs, P.perm, P.listed, P.ids, P.runs, P.many, P.part}) printf(" %zu", o);
  printf("\n");
}"""


def test_embedding_regions(tmp_path):
    run = program(tmp_path, EMBED)
    for vocab, dim in ((1, 1), (5, 300), (511, 7), (1 << 20, 1 << 18), (152064, 3584)):
        assert run(4096, vocab, dim)[0][3] == "256"
        most = 0
        for n in (4097, 5000, 65535, 65536, 65537, 66000, 1 << 24, (1 << 31) - 1):
            tiles, tile, runs, total, *at = map(int, run(n, vocab, dim)[0])
            buckets = min(512, 1 << (vocab - 1).bit_length())
            assert tiles <= 64 and (tiles - 1) * tile < n <= tiles * tile
            # ids with m > 32 tokens take ceil(m / 32) runs: most of them where every id has 33
            assert runs >= n // 33 * 2
            sizes = [4 * tiles, 4 * tiles * buckets, 4 * (buckets + 1), 8 * n, 4 * n, 4 * 32 * 17, 16 * n, 8 * runs,
                     16 * (n // 33), 4 * runs * dim]
            assert at[0] >= 256 and all(o % 256 == 0 for o in at)
            for o, size, end in zip(at, sizes, at[1:] + [total]):
                assert o + size <= end
            assert total >= most
            most = total


GROUPS = r"""int main(int n, char** v) {
  std::vector<iso_weight_grad> g((n - 2) / 3);
  for (size_t j = 0; j < g.size(); ++j)
    g[j].grad = (void*)(uintptr_t)atoll(v[2 + 3 * j]), g[j].rows = atoll(v[3 + 3 * j]), g[j].in.cols = atoll(v[4 + 3 * j]);
  printf("%d\n", weight_grad_group(g.data(), (int)g.size(), atoi(v[1])));
}"""


def test_layers_of_one_launch(tmp_path):
    """A launch ends before a gradient that shares memory with one of its own, and after 16 layers."""
    run = program(tmp_path, GROUPS)
    apart = [(4096 * (j + 1), 16, 64) for j in range(20)]          # 4096 bytes each in fp32, 2048 in bf16

    def group(layers, dt=0):
        return int(run(dt, *[w for l in layers for w in l])[0][0])
    assert group([]) == 0 and group(apart[:1]) == 1 and group(apart[:9]) == 9 and group(apart) == 16
    for dt in (0, 1):
        assert group(apart[:5] + apart[2:3] + apart[6:9], dt) == 5          # the same
        assert group(apart[:2] + apart[:1] * 3, dt) == 2
    part = [(4096, 16, 64), (4096 + 2048, 16, 64)]                 # the second half of the first in fp32, behind it in bf16
    assert group(part, 0) == 1 and group(part[::-1], 0) == 1 and group(part, 1) == 2
    assert group([(4096, 16, 64), (4096, 0, 64), (5000, 16, 0), (8192, 1, 1)]) == 4    # empty ones share nothing
    assert group([(4096, 1 << 24, 1 << 10), (4096 + (1 << 35), 4, 4)]) == 1            # past 32 bits


def test_who_looks_at_the_ids(tmp_path):
    """Up to 6144 tokens one workgroup, up to 16384 where rows are long enough for the copies to outlast it."""
    run = program(tmp_path, 'int main(int, char** v) { printf("%d\\n", lookup_checks_alone(atoll(v[1]), atoll(v[2]))); }')
    for row, most in ((2, 6144), (128, 6144), (4096, 6144), (4098, 16384), (7168, 16384), (1 << 20, 16384)):
        for tokens, alone in ((0, 1), (1, 1), (6144, 1), (most, 1), (most + 1, 0), (1 << 31, 0)):
            assert run(tokens, row) == [[str(alone)]], (tokens, row)
