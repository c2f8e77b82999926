"""iso_attend and iso_attend_grad: head layouts, many sequences, offsets past 32 bits, calls side by side; and a run of the
training operators from the embedding to the weight gradients.  The bounds are those of tests/attn_helpers.py."""
import numpy as np
import pytest

import paper_2607_19331_amd as iso
from tests.attn_helpers import Case
from tests.grad_helpers import code, ttype
from tests.gpu_helpers import say

pytestmark = pytest.mark.gpu


def run(case):
    ws = case.forward()
    assert iso.iso_read_device_status(ws) == 0
    case.check_forward()
    ws = case.backward()
    assert iso.iso_read_device_status(ws) == 0
    case.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("heads,kv,dim", [(3, 3, 16), (5, 5, 72), (6, 3, 128), (8, 8, 8), (16, 16, 32), (20, 4, 64), (33, 1, 64), (40, 1, 24),
                                          (200, 1, 8), (1024, 1, 8)])
def test_head_layouts(dtype, heads, kv, dim):
    say(f"attend heads {dtype} {heads}/{kv} x {dim}")
    lens = [37, 5] if heads <= 64 else [6, 3]
    run(Case(dtype, lens, lens, heads, kv, dim, True, gap=8))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [63, 64, 65, 200])
def test_many_sequences(dtype, n):
    """More sequences than a wave has lanes, some of them empty."""
    say(f"attend sequences {dtype} {n}")
    rng = np.random.default_rng(n)
    q, k = rng.integers(0, 12, n).tolist(), rng.integers(0, 30, n).tolist()
    q[n // 2], k[n // 2] = 90, 140
    run(Case(dtype, q, k, 2, 1, 16, True))
    run(Case(dtype, [min(x, 1) for x in q], [7 * x for x in k], 4, 2, 32, True))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("q,k,window,causal", [([1], [9000], 0, True), ([3], [4001], 0, False), ([1, 2], [700, 6000], 1000, True),
                                               ([2000], [3], 0, False), ([1500], [1500], 40, True), ([60, 600], [1200, 600], 0, True)])
def test_long_walks_shared_out(dtype, q, k, window, causal):
    """Few tiles whose keys or rows are many: pieces and their joins, some with nothing to do."""
    say(f"attend pieces {dtype} {q} {k} {window}")
    run(Case(dtype, q, k, 2, 1, 64, causal, window))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("window", [70, 1 << 30, (1 << 31) + 5, 1 << 62, (1 << 63) - 1])
def test_windows_wider_than_a_sequence(window, causal):
    say(f"attend window {window} {causal}")
    run(Case("f32", [33, 9], [70, 3], 2, 1, 16, causal, window))


def test_partial_sums_stay_in_the_workspace():
    """3199 rows over 400000 keys: 25 tiles of 64 pieces, the most that a workspace has to hold."""
    import torch
    say("attend workspace's end")
    tokens, keys, heads, dim = 457, 400000, 7, 8
    g = torch.Generator("cuda").manual_seed(3)
    new = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    dev = lambda n: torch.tensor([0, n], dtype=torch.int32, device="cuda")  # noqa: E731
    q, k, v, dout = new(tokens, heads * dim), new(keys, dim), new(keys, dim), new(tokens, heads * dim)
    a = iso.Attn(q=q, k=k, v=v, ld_q=heads * dim, ld_k=dim, ld_v=dim, start_q=dev(tokens), start_k=dev(keys), sequences=1,
                 tokens_q=tokens, tokens_k=keys, heads=heads, heads_kv=1, dim=dim, scale=0.3, causal=False, window=0,
                 out=torch.empty_like(q), ld_out=heads * dim, lse=torch.empty(tokens, heads, device="cuda"), dout=dout, ld_dout=heads * dim,
                 dq=torch.empty_like(q), dk=torch.empty_like(k), dv=torch.empty_like(v), ld_dq=heads * dim, ld_dk=dim, ld_dv=dim)
    for grad, call in ((False, iso.iso_attend), (True, iso.iso_attend_grad)):
        size = iso.attend_workspace(a, iso.F32, grad).numel()
        ws = torch.full((size + (1 << 23),), 0x5A, dtype=torch.uint8, device="cuda")
        call(a, iso.F32, ws=ws[:size])
        assert iso.iso_read_device_status(ws) == 0
        assert bool((ws[size:] == 0x5A).all())
    # The first query's row.  A lane adds up 3200 terms at most in binary32, with pieces and halves: 3300 2^-24 of a sum of weights
    # times |v| (below 1); scores are off by 16 2^-24 times 20: together below 3e-4.
    x = (k.double() @ q[0, :dim].double()) * 0.3
    want = torch.softmax(x, 0) @ v.double()
    assert torch.allclose(a.out[0, :dim].double(), want, rtol=0, atol=3e-4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,heads,kv,causal", [([3000, 700, 0, 130], 4, 1, True),          # 94 tiles a sequence and more than 64 places
                                                  ([2600, 1300, 1000], 8, 8, True),           # 40 tiles a head for 32 CUs: all start at once
                                                  ([700, 1300, 500], 16, 16, False),          # two heads of 21 tiles each
                                                  ([1, 900, 2, 900, 3] * 12, 8, 4, True)])    # 60 sequences
def test_order_of_tiles(dtype, lens, heads, kv, causal):
    say(f"attend order {dtype} {lens} {heads}/{kv}")
    run(Case(dtype, lens, lens, heads, kv, 16, causal))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_non_finite_values_in_pieces(dtype):
    say(f"attend pieces non-finite {dtype}")

    def edit(case):   # the last keys of 3000, which the last query alone sees
        case.host["v"][int(case.at_k[-1]) - 1] = np.inf
        case.host["k"][int(case.at_k[-1]) - 1, 0] = np.nan
    case = Case(dtype, [4], [3000], 2, 1, 64, True, edit=edit)
    case.forward()
    out = case.out.host()[int(case.at_q[0]):int(case.at_q[-1])]
    assert np.isfinite(out[:-1]).all() and not np.isfinite(out[-1]).any()
    case.backward()
    s = slice(int(case.at_q[0]), int(case.at_q[-1]) - 1)
    assert np.isfinite(case.dq.host()[s]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_past_32_bits(dtype):
    """Strides of 2^21 elements: rows of one sequence lie 4.5 GB (bf16) and 9 GB apart."""
    import torch
    n, ld, dim = 1090, iso._lib.ATTN_MAX_LD, 16
    say(f"attend wide strides {dtype}")
    small = Case(dtype, [n], [n], 2, 1, dim, True, 64, before=0)
    small.forward(), small.backward()
    a, t, hold = small.a, ttype(dtype), {}
    rows = a.tokens_q
    for name in ("q", "k", "v", "out", "dout", "dq", "dk", "dv"):
        buf = hold[name] = torch.empty(rows * ld, dtype=t, device="cuda").view(rows, ld)
        if name in ("q", "k", "v", "dout"):
            src = getattr(small, name).view
            buf[:, :src.shape[1]] = src
        setattr(a, name, buf)
        setattr(a, "ld_" + name, ld)
    small.lse.view.fill_(7.25)
    ws = iso.attend_workspace(a, code(dtype))
    iso.iso_attend(a, code(dtype), ws=ws)
    ws = iso.attend_workspace(a, code(dtype), grad=True)
    iso.iso_attend_grad(a, code(dtype), ws=ws)
    assert iso.iso_read_device_status(ws) == 0
    for name in ("out", "dq", "dk", "dv"):
        m = getattr(small, name)
        assert torch.equal(hold[name][:n, :m.cols], m.view[:n]), name
    del hold
    torch.cuda.empty_cache()


def test_a_long_cache():
    """The last of 2.2 million keys (4.5 GB of each of k and v), all others of no sequence."""
    import torch
    say("attend long cache")
    n, m, tokens = 3, 900, 2200000
    small = Case("bf16", [n], [m], 16, 8, 128, True, before=0)
    small.forward()
    a = small.a
    want = small.out.view[:n].clone()
    hold = [torch.empty(tokens, 8 * 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for buf, x in zip(hold, (small.k, small.v)):
        buf[tokens - m:] = x.view[:m]
    a.k, a.v, a.ld_k, a.ld_v, a.tokens_k = hold[0], hold[1], 1024, 1024, tokens
    a.start_k = torch.tensor([tokens - m, tokens], dtype=torch.int32, device="cuda")
    small.out.view.fill_(7.25)
    ws = iso.attend_workspace(a, iso.BF16)
    iso.iso_attend(a, iso.BF16, ws=ws)
    assert iso.iso_read_device_status(ws) == 0
    # other pieces than those of the small call: the same sums in another order, each rounded to bf16 once
    got = small.out.view[:n]
    assert torch.allclose(got.float(), want.float(), rtol=2.0 ** -6, atol=2.0 ** -7)
    small.check_forward()
    del hold
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_calls_side_by_side(dtype):
    """Two streams, a workspace each, no wait between them."""
    import torch
    say(f"attend two streams {dtype}")
    cases = [Case(dtype, [400, 33], [400, 33], 6, 2, 64, True, seed=s) for s in (1, 2)]
    spaces = [(iso.attend_workspace(c.a, code(dtype)), iso.attend_workspace(c.a, code(dtype), grad=True)) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(3):
        for c, (f, b), s in zip(cases, spaces, streams):
            c.forward(f, s), c.backward(b, s)
    torch.cuda.synchronize()
    for c in cases:
        c.check_forward(), c.check_backward()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_training_step_of_the_operators(dtype):
    """Embedding -> q, k, v -> attention -> logits -> distillation, and back to every weight gradient, against autograd in
    binary64 on the same rounded values.  Bound: activations and gradients are rounded to the type at every operator (about ten
    roundings one after another), checkpoints keep 8 bits; 6% of a gradient's norm covers them in bf16, 2% in fp32, whose
    weight gradients read the 8-bit checkpoints too."""
    import torch
    say(f"training step {dtype}")
    g = torch.Generator().manual_seed(3)
    dt, t, f64 = code(dtype), ttype(dtype), torch.float64
    vocab, dim, heads, kv, hd, top, temp = 211, 64, 4, 2, 16, 6, 2.0
    lens = [40, 1, 23]
    n = sum(lens)
    wide, narrow = heads * hd, kv * hd
    rnd = lambda *s, f=1.0: (torch.randn(*s, generator=g, dtype=f64) * f).to(t).cuda()  # noqa: E731
    emb, wqkv, wo = rnd(vocab, dim), rnd(wide + 2 * narrow, dim, f=dim ** -0.5), rnd(vocab, wide, f=wide ** -0.5)
    ids = torch.randint(0, vocab, (n,), generator=g).cuda()
    tids, ty = torch.randint(0, vocab, (n, top), generator=g).cuda(), torch.randn(n, top, generator=g).cuda() * 2
    weight = (torch.rand(n, generator=g) / n).cuda()
    start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    new = lambda *s: torch.zeros(*s, dtype=t, device="cuda")  # noqa: E731

    e = iso.Embed(ids=ids, tokens=n, vocab=vocab, dim=dim, x=new(n, dim), table=emb, grad=new(vocab, dim))
    ews = iso.embed_workspace(e)
    iso.iso_embed_lookup(e, dt, ws=ews)
    x = e.x
    qkv, dqkv = x @ wqkv.t(), new(n, wide + 2 * narrow)
    cols = (slice(0, wide), slice(wide, wide + narrow), slice(wide + narrow, None))
    ld = qkv.stride(0)
    a = iso.Attn(q=qkv[:, cols[0]], k=qkv[:, cols[1]], v=qkv[:, cols[2]], ld_q=ld, ld_k=ld, ld_v=ld, start_q=start, start_k=start,
                 sequences=len(lens), tokens_q=n, tokens_k=n, heads=heads, heads_kv=kv, dim=hd, scale=hd ** -0.5, causal=True,
                 out=new(n, wide), lse=torch.zeros(n, heads, device="cuda"))
    fws = iso.attend_workspace(a, dt)
    iso.iso_attend(a, dt, ws=fws)
    logits = a.out @ wo.t()
    kept = []
    for y in (x, a.out):
        c = iso.Ckpt(n, y.shape[1], *iso.ckpt_buffers(n, y.shape[1]), x=y, ld_x=y.stride(0))
        iso.iso_ckpt_pack([c], dt)
        kept.append(c)
    d = iso.Distill(logits=logits, tokens=n, vocab=vocab, ids=tids, teacher=ty, top=top, loss=torch.zeros(n, device="cuda"),
                    lse=torch.zeros(n, device="cuda"), grad=logits, weight=weight, temperature=temp)
    dws = iso.distill_workspace(d)
    iso.iso_distill_loss(d, dt, ws=dws)
    dlogits = logits                                   # the gradient lies over the logits
    a.dout, a.ld_dout = dlogits @ wo, wide
    a.dq, a.dk, a.dv = (dqkv[:, c] for c in cols)
    a.ld_dq = a.ld_dk = a.ld_dv = ld
    bws = iso.attend_workspace(a, dt, grad=True)
    iso.iso_attend_grad(a, dt, ws=bws)
    gwo, gqkv = new(vocab, wide), new(wide + 2 * narrow, dim)
    jobs = [iso.WeightGrad(kept[1], dy=dlogits, grad=gwo, rows=vocab), iso.WeightGrad(kept[0], dy=dqkv, grad=gqkv, rows=wide + 2 * narrow)]
    iso.iso_ckpt_weight_grad(jobs, dt, dt, ws=iso.weight_grad_workspace(jobs, dt))
    e.x = dqkv @ wqkv
    iso.iso_embed_grad(e, dt, dt, ws=ews)
    for ws in (ews, fws, dws, bws):
        assert iso.iso_read_device_status(ws) == 0

    E, W, O = (w.double().cpu().requires_grad_() for w in (emb, wqkv, wo))
    X = E[ids.cpu()]
    Q, K, V = (X @ W.t()).split([wide, narrow, narrow], 1)
    outs, at = [], 0
    for m in lens:
        q = Q[at:at + m].view(m, kv, heads // kv, hd)
        k, v = (y[at:at + m].view(m, kv, hd) for y in (K, V))
        s = torch.stack([torch.stack([q[:, h, r] @ k[:, h].t() for r in range(heads // kv)]) for h in range(kv)]) * hd ** -0.5
        s = s.masked_fill(torch.triu(torch.ones(m, m, dtype=torch.bool), 1), -np.inf)
        o = torch.stack([torch.stack([torch.softmax(s[h, r], 1) @ v[:, h] for r in range(heads // kv)], 1) for h in range(kv)], 1)
        outs.append(o.reshape(m, wide))
        at += m
    Z = torch.cat(outs) @ O.t() / temp
    share = torch.softmax(ty.cpu().double() / temp, 1)
    logp = torch.log_softmax(Z, 1).gather(1, tids.cpu())
    losses = weight.cpu().double() * temp ** 2 * (share * (torch.log(share) - logp)).sum(1)
    losses.sum().backward()
    assert abs(float(d.loss.double().sum()) - float(losses.sum().detach())) < 0.02 * abs(float(losses.sum().detach()))
    for got, want in ((e.grad, E.grad), (gqkv, W.grad), (gwo, O.grad)):
        off = float((got.double().cpu() - want).norm() / want.norm())
        assert off < (0.06 if dtype == "bf16" else 0.02), off
