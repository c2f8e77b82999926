"""Attention and distillation, forward and backward: inputs, one pass, minimal work, 64-bit reference.

A case is a dict of plain values.  `kind` names the entry point it goes through:

  attend   iso_attend          O = softmax(scale Q K^T) V over the keys that a query may see, and the log-sum-exp of its scores
  agrad    iso_attend_grad     dQ, dK, dV from Q, K, V, O, the log-sum-exp and dO, the probabilities recomputed
  loss     iso_distill_loss    w T^2 KL(teacher's top entries || student) per token, and the log-sum-exp of its logits / T
  both     iso_distill_loss    the same with the logits' gradient, in one call
  dgrad    iso_distill_grad    the logits' gradient w T (softmax(z / T) - teacher) from the kept log-sum-exp

Attention runs over packed sequences: `lens_q` and `lens_k` list their numbers of queries and keys ("3*512,17" is 512, 512,
512, 17), rows lie one after another.  Query i of a sequence with n queries and m keys stands at position p = i + m - n.  It sees
keys up to p where `causal`, only those nearer than `window` to p where that is not 0.  A query that sees no key has a zero
result and minus infinity as log-sum-exp.  `heads` query heads share `kv` key and value heads in consecutive groups.  With
`packed`, q, k and v (and their gradients) are column ranges of one buffer, as one projection leaves them.

A teacher's entry is an id and a logit; id -1 is none.  A token without entries, or with weight 0, adds nothing.
"""
import math

import torch

own = False

DEV = "cuda"


# ---- the listed cases and the ranges they stand for ----------------------------------------------------------------

RAGGED = "2048,31,700,1999,5,1024,333,1500,64,1,1777,900,129,257,2000,611"
CACHED = "8192,513,4000,77,6001,1024,2500,8191,300,3333,4096,1,7000,129,5120,900"


def listed():
    return [
        # fp32 training of a tiny model with odd lengths and heads of 40: a call whose cost is its launch
        dict(name="attend_small_f32", kind="attend", dtype="f32", lens_q="5,1,37", lens_k="5,1,37", heads=6, kv=2, dim=40,
             causal=True, window=0, packed=True),
        # one new token for each of 16 rollouts of different lengths, the 7B head layout
        dict(name="attend_token_bf16", kind="attend", dtype="bf16", lens_q="16*1", lens_k=CACHED, heads=28, kv=4, dim=128,
             causal=True, window=0, packed=False),
        # 16 packed samples of ragged lengths through a layer with a sliding window and heads of 64
        dict(name="attend_window_bf16", kind="attend", dtype="bf16", lens_q=RAGGED, lens_k=RAGGED, heads=16, kv=4, dim=64,
             causal=True, window=512, packed=True),
        # a micro-batch of four full sequences through a 7B layer
        dict(name="attend_7b_bf16", kind="attend", dtype="bf16", lens_q="4*4096", lens_k="4*4096", heads=28, kv=4, dim=128,
             causal=True, window=0, packed=True),
        # fp32 gradients of a small model, every query sees every key
        dict(name="agrad_small_f32", kind="agrad", dtype="f32", lens_q="11,64,3", lens_k="11,64,3", heads=3, kv=3, dim=64,
             causal=False, window=0, packed=True),
        # packed samples of ragged lengths through a 1.5B layer
        dict(name="agrad_ragged_bf16", kind="agrad", dtype="bf16", lens_q=RAGGED, lens_k=RAGGED, heads=12, kv=2, dim=128,
             causal=True, window=0, packed=True),
        # two long sequences through a 7B layer
        dict(name="agrad_long_bf16", kind="agrad", dtype="bf16", lens_q="2*8192", lens_k="2*8192", heads=28, kv=4, dim=128,
             causal=True, window=0, packed=True),
        # one token over the 1.5B vocabulary: one row for the whole card
        dict(name="loss_token_bf16", kind="loss", dtype="bf16", ids="i64", tokens=1, vocab=151936, top=20, temp=1.0, pad=False,
             gap=0),
        # the loss alone of a 7B batch (validation)
        dict(name="loss_7b_bf16", kind="loss", dtype="bf16", ids="i64", tokens=4096, vocab=152064, top=64, temp=2.0, pad=True,
             gap=0),
        # a small odd vocabulary with strided rows
        dict(name="dgrad_small_f32", kind="dgrad", dtype="f32", ids="i32", tokens=7, vocab=1031, top=5, temp=1.0, pad=True, gap=3),
        # the backward pass of a 7B batch whose forward pass kept the log-sum-exp
        dict(name="dgrad_7b_bf16", kind="dgrad", dtype="bf16", ids="i64", tokens=4096, vocab=152064, top=64, temp=2.0, pad=True,
             gap=0),
        # loss and gradient at once, as a training step takes them
        dict(name="both_7b_bf16", kind="both", dtype="bf16", ids="i64", tokens=4096, vocab=152064, top=64, temp=2.0, pad=True,
             gap=0),
    ]


MOST_PAIRS = 28 * 8192 * 8192 // 2     # heads times pairs of padded lengths, a drawn case
MOST_LOGITS = 1 << 29


def draw(rng):
    def logint(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["attend", "attend", "attend", "agrad", "agrad", "agrad", "loss", "both", "dgrad"])
    c = dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]))
    if kind in ("loss", "both", "dgrad"):
        c.update(ids=rng.choice(["i64", "i32"]), tokens=logint(1, 8192), vocab=logint(64, 152064), temp=rng.choice([1.0, 2.0, 0.7]),
                 pad=rng.choice([True, False]), gap=rng.choice([0, 0, 8, 64, 3]))
        c["tokens"] = min(c["tokens"], MOST_LOGITS // c["vocab"])
        c["top"] = logint(1, min(256, c["vocab"]))
        return c
    kv = rng.choice([1, 2, 2, 4, 8])
    c.update(kv=kv, heads=kv * rng.choice([1, 1, 2, 4, 6, 7, 8]), dim=rng.choice([64, 64, 128, 128, 128, 8 * rng.randint(1, 16)]),
             causal=rng.random() < 0.8, window=rng.choice([0, 0, 0, logint(8, 2048)]), packed=rng.choice([True, False]))
    # whole samples, new tokens after kept ones, one new token a sequence, and now and then fewer keys than queries
    style = rng.choice(["whole", "whole", "whole", "after", "after", "one", "fewer"])
    longest, n = logint(16, 8192), logint(1, 64)
    most = MOST_PAIRS // (c["heads"] * (1 if c["dtype"] == "bf16" else 8))
    while n > 1 and n * longest * (1 if style == "one" else longest) > most:
        n //= 2
    while n * longest * (1 if style == "one" else longest) > most:
        longest = longest * 3 // 4
    m = [longest if at == 0 or rng.random() < 0.3 else logint(1, longest) for at in range(n)]
    q = {"whole": m, "after": [logint(1, x) for x in m], "one": [1] * n, "fewer": [min(longest, x + rng.randint(0, 5)) for x in m]}[style]
    c.update(lens_q=",".join(str(x) for x in q), lens_k=",".join(str(x) for x in m))
    return c


def _lens(text):
    """'2*3,4' -> [3, 3, 4]."""
    out = []
    for part in text.split(","):
        times, one = part.split("*") if "*" in part else ("1", part)
        out += [int(one)] * int(times)
    return out


# ---- inputs --------------------------------------------------------------------------------------------------------

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _starts(lens):
    at = [0]
    for x in lens:
        at.append(at[-1] + x)
    return torch.tensor(at, dtype=torch.int32, device=DEV)


def _columns(case, dt, nq, nk):
    """Buffers for q, k, v: column ranges of one where they are packed and have the same rows."""
    a, b = case["heads"] * case["dim"], case["kv"] * case["dim"]
    if case["packed"] and nq == nk:
        buf = torch.zeros(nq, a + 2 * b, dtype=dt, device=DEV)
        return buf[:, :a], buf[:, a:a + b], buf[:, a + b:]
    return tuple(torch.zeros(n, w, dtype=dt, device=DEV) for n, w in ((nq, a), (nk, b), (nk, b)))


def prepare(case, seed):
    g, dt = torch.Generator(device=DEV).manual_seed(seed), _type(case["dtype"])

    def normal(*shape):
        return torch.randn(*shape, generator=g, device=DEV)

    s = dict(case=case)
    if case["kind"] in ("attend", "agrad"):
        lq, lk = _lens(case["lens_q"]), _lens(case["lens_k"])
        nq, nk, heads, kv, dim = sum(lq), sum(lk), case["heads"], case["kv"], case["dim"]
        s["start_q"], s["start_k"], s["scale"] = _starts(lq), _starts(lk), 1.0 / math.sqrt(dim)
        s["q"], s["k"], s["v"] = _columns(case, dt, nq, nk)
        # scores as a trained layer's: wide enough that a few keys take most of a row, and a bias common to all keys
        s["q"].copy_(1.5 * normal(nq, heads * dim))
        s["k"].copy_(normal(nk, kv * dim) + 2.0 * normal(kv * dim))
        s["v"].copy_(normal(nk, kv * dim))
        s["out"] = torch.zeros(nq, heads * dim, dtype=dt, device=DEV)
        s["lse"] = torch.zeros(nq, heads, device=DEV)
        if case["kind"] == "agrad":
            s["dout"] = (1e-2 * normal(nq, heads * dim)).to(dt)
            s["dq"], s["dk"], s["dv"] = _columns(case, dt, nq, nk)
            out, lse = _attend(s)
            s["out"].copy_(out)
            s["lse"].copy_(lse)
        return s
    n, vocab, top, gap = case["tokens"], case["vocab"], case["top"], case["gap"]
    idt = torch.int64 if case["ids"] == "i64" else torch.int32
    first = torch.randint(0, vocab, (n, 1), generator=g, device=DEV)
    step = torch.randint(1, max(2, vocab // top + 1), (n, 1), generator=g, device=DEV)
    ids = (first + step * torch.arange(top, device=DEV)) % vocab  # different ids: step * top <= vocab
    # the teacher's logits fall from its first entry on; the student has learnt about the same
    s["teacher"] = (3.0 * normal(n, top)).sort(1, descending=True)[0] + 12.0
    z = torch.zeros(n, vocab + gap, dtype=dt, device=DEV)
    z[:, :vocab] = (2.0 * normal(n, vocab)).scatter_(1, ids, s["teacher"] + normal(n, top)).to(dt)
    s["z"] = z[:, :vocab]
    s["weight"] = torch.full((n,), 1.0 / n, device=DEV)
    if case["pad"]:  # shorter lists, and tokens that do not count
        have = torch.randint(1, top + 1, (n, 1), generator=g, device=DEV)
        ids = torch.where(torch.arange(top, device=DEV) < have, ids, -1)
        s["weight"] *= torch.rand(n, generator=g, device=DEV) < 0.8
    s["ids"] = ids.to(idt)
    s["loss"], s["lse"] = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    if case["kind"] != "loss":
        s["grad"] = torch.zeros(n, vocab + gap, dtype=dt, device=DEV)[:, :vocab]
    if case["kind"] == "dgrad":
        s["lse"].copy_(_lse(s["z"].float() / case["temp"]))
    return s


# ---- one pass ------------------------------------------------------------------------------------------------------

def run(s):
    return _run_own(s) if own else _run_plain(s)


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "attend":
        return list(_attend(s))
    if kind == "agrad":
        return list(_attend_grad(s))
    return _distill(s)


def _padded(x, start, longest, heads):
    """Packed rows (rows x heads * dim) as sequences x heads x longest x dim in 32 bits, zeros behind each sequence."""
    at = start[:-1, None].long() + torch.arange(longest, device=DEV)
    live = at < start[1:, None]
    rows = x.float()[at.clamp(max=x.shape[0] - 1)] * live[:, :, None]
    return rows.view(*at.shape, heads, -1).transpose(1, 2).contiguous()


def _unpadded(x, start, rows, dt):
    """The inverse of _padded."""
    at = torch.arange(rows, dtype=torch.int32, device=DEV)
    seq = torch.searchsorted(start[1:].contiguous(), at, right=True)
    return x.transpose(1, 2)[seq, at.long() - start[seq].long()].reshape(rows, -1).to(dt)


def _grouped(s):
    """Queries as sequences x kv x (group * queries) x dim, keys, values, and which keys a query may see."""
    case = s["case"]
    kv, dim = case["kv"], case["dim"]
    lq, lk = _lens(case["lens_q"]), _lens(case["lens_k"])
    m, n = max(lq), max(lk)
    q = _padded(s["q"], s["start_q"], m, case["heads"]).view(len(lq), kv, -1, dim)
    k, v = (_padded(s[x], s["start_k"], n, kv) for x in ("k", "v"))
    nq, nk = (s[x][1:, None, None] - s[x][:-1, None, None] for x in ("start_q", "start_k"))
    i, j = torch.arange(m, device=DEV)[:, None], torch.arange(n, device=DEV)
    p = i + nk - nq
    see = (j < nk) & (i < nq)
    if case["causal"]:
        see = see & (j <= p)
    if case["window"]:
        see = see & (j > p - case["window"]) & (j < p + case["window"])
    return q, k, v, see.repeat(1, case["heads"] // kv, 1)[:, None]


def _attend(s):
    case, dt, nq = s["case"], _type(s["case"]["dtype"]), s["q"].shape[0]
    q, k, v, see = _grouped(s)
    x = (q @ k.transpose(2, 3)).mul_(s["scale"]).masked_fill_(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(top.clamp(min=torch.finfo(torch.float32).min)).exp_()
    total = x.sum(-1, keepdim=True)
    out = (x @ v) / total.clamp(min=1.0)
    lse = top + torch.log(total)
    heads, n = case["heads"], len(_lens(case["lens_q"]))
    return (_unpadded(out.view(n, heads, -1, case["dim"]), s["start_q"], nq, dt),
            _unpadded(lse.view(n, heads, -1, 1), s["start_q"], nq, torch.float32))


def _attend_grad(s):
    case, dt, nq, nk = s["case"], _type(s["case"]["dtype"]), s["q"].shape[0], s["k"].shape[0]
    heads, kv, dim, m = case["heads"], case["kv"], case["dim"], max(_lens(case["lens_q"]))
    q, k, v, see = _grouped(s)
    n = q.shape[0]
    dout, out = (_padded(s[x], s["start_q"], m, heads).view(n, kv, -1, dim) for x in ("dout", "out"))
    lse = _padded(s["lse"], s["start_q"], m, heads).view(n, kv, -1, 1)
    p = (q @ k.transpose(2, 3)).mul_(s["scale"]).sub_(lse).masked_fill_(~see, -math.inf).exp_()
    dv = p.transpose(2, 3) @ dout
    ds = (dout @ v.transpose(2, 3)).sub_((dout * out).sum(-1, keepdim=True)).mul_(p).mul_(s["scale"])
    dq, dk = ds @ k, ds.transpose(2, 3) @ q
    return (_unpadded(dq.view(n, heads, -1, dim), s["start_q"], nq, dt), _unpadded(dk, s["start_k"], nk, dt),
            _unpadded(dv, s["start_k"], nk, dt))


def _lse(z):
    top = z.amax(1)
    return top + torch.log(torch.exp(z - top[:, None]).sum(1))


def _distill(s):
    case, kind, temp = s["case"], s["case"]["kind"], s["case"]["temp"]
    z, ids, have = s["z"].float() / temp, s["ids"].long().clamp(min=0), s["ids"] >= 0
    x = torch.where(have, s["teacher"] / temp, -math.inf)
    log_t = x - _lse(x)[:, None]
    t = torch.exp(log_t)
    out = []
    lse = s["lse"] if kind == "dgrad" else _lse(z)
    if kind != "dgrad":
        part = torch.where(have, t * (log_t - (z.gather(1, ids) - lse[:, None])), 0.0)
        out += [s["weight"] * temp * temp * part.sum(1), lse]
    if kind != "loss":
        dz = torch.exp(z - lse[:, None]).scatter_add_(1, ids, -t)
        out.append((dz * (s["weight"] * temp)[:, None]).to(_type(case["dtype"])))
    return out


def _run_own(s):
    import paper_2607_19331_amd as iso

    case, kind = s["case"], s["case"]["kind"]
    dt = {"bf16": iso.BF16, "f32": iso.F32}[case["dtype"]]
    if kind in ("attend", "agrad"):
        a = iso.Attn(q=s["q"], k=s["k"], v=s["v"], ld_q=s["q"].stride(0), ld_k=s["k"].stride(0), ld_v=s["v"].stride(0),
                     start_q=s["start_q"], start_k=s["start_k"], sequences=s["start_q"].numel() - 1, tokens_q=s["q"].shape[0],
                     tokens_k=s["k"].shape[0], heads=case["heads"], heads_kv=case["kv"], dim=case["dim"], scale=s["scale"],
                     causal=case["causal"], window=case["window"], out=s["out"], lse=s["lse"])
        if kind == "agrad":
            a.dout, a.dq, a.dk, a.dv = s["dout"], s["dq"], s["dk"], s["dv"]
            a.ld_dq, a.ld_dk, a.ld_dv = s["dq"].stride(0), s["dk"].stride(0), s["dv"].stride(0)
        if "ws" not in s:  # a program keeps its workspace
            s["ws"] = iso.attend_workspace(a, dt, grad=kind == "agrad", device=DEV)
        if kind == "attend":
            iso.iso_attend(a, dt, ws=s["ws"])
            return [s["out"], s["lse"]]
        iso.iso_attend_grad(a, dt, ws=s["ws"])
        return [s["dq"], s["dk"], s["dv"]]
    d = iso.Distill(logits=s["z"], tokens=case["tokens"], vocab=case["vocab"], ld=s["z"].stride(0), ids=s["ids"],
                    teacher=s["teacher"], top=case["top"], pad_id=-1, weight=s["weight"], temperature=case["temp"], loss=s["loss"],
                    lse=s["lse"])
    if kind != "loss":
        d.grad, d.ld_grad = s["grad"], s["grad"].stride(0)
    if "ws" not in s:
        s["ws"] = iso.distill_workspace(d, DEV)
    if kind == "dgrad":
        iso.iso_distill_grad(d, dt, ws=s["ws"])
        return [s["grad"]]
    iso.iso_distill_loss(d, dt, ws=s["ws"])
    return [s["loss"], s["lse"]] + ([s["grad"]] if kind == "both" else [])


# ---- minimal work and the 64-bit reference -------------------------------------------------------------------------

def _size(name):
    return 2 if name == "bf16" else 4


def _seen(case):
    """How many (query, key) pairs count."""
    total = 0
    for n, m in zip(_lens(case["lens_q"]), _lens(case["lens_k"])):
        p = torch.arange(n, dtype=torch.int64) + (m - n)
        w = case["window"] or max(n, m) + m + 1
        last = torch.clamp(p if case["causal"] else p + w - 1, max=m - 1)
        total += int((last - torch.clamp(p - w + 1, min=0) + 1).clamp(min=0).sum())
    return total


def work(case):
    kind, size = case["kind"], _size(case["dtype"])
    if kind in ("attend", "agrad"):
        nq, nk, dim = sum(_lens(case["lens_q"])), sum(_lens(case["lens_k"])), case["dim"]
        a, b = nq * case["heads"] * dim * size, nk * case["kv"] * dim * size
        pairs = case["heads"] * _seen(case)
        if kind == "attend":
            return {"bytes": 2 * a + 2 * b + nq * case["heads"] * 4, "flops": 4.0 * dim * pairs}
        return {"bytes": 4 * a + 4 * b + nq * case["heads"] * 4, "flops": 10.0 * dim * pairs}
    n, vocab = case["tokens"], case["vocab"]
    lists = n * case["top"] * (4 + (8 if case["ids"] == "i64" else 4)) + 12 * n
    return {"bytes": n * vocab * size * (1 if kind == "loss" else 2) + lists, "flops": n * vocab * (8.0 if kind == "both" else 4.0)}


def exact(case, seed):
    """From the definitions, in binary64 on the inputs of prepare(case, seed): one sequence and head at a time, one token's
    row of logits at a time in blocks."""
    s, kind = prepare(case, seed), case["kind"]
    if kind in ("attend", "agrad"):
        return _exact_attention(s, case)
    temp, out = case["temp"], [[], [], []]
    for lo in range(0, case["tokens"], 512):
        cut = slice(lo, lo + 512)
        z = s["z"][cut].double() / temp
        lse = s["lse"][cut].double() if kind == "dgrad" else torch.logsumexp(z, 1)
        t = torch.zeros(z.shape[0], z.shape[1] + 1, dtype=torch.float64, device=DEV)  # entries without an id in the last column
        ids = torch.where(s["ids"][cut] < 0, z.shape[1], s["ids"][cut]).long()
        x = torch.where(s["ids"][cut] < 0, -math.inf, s["teacher"][cut].double() / temp)
        t.scatter_(1, ids, torch.softmax(x, 1))
        t = t[:, :-1]
        w = s["weight"][cut].double()
        if kind != "dgrad":
            kl = torch.special.xlogy(t, t).sum(1) - (t * z).sum(1) + lse
            out[0].append(w * temp ** 2 * kl)
            out[1].append(lse)
        if kind != "loss":
            out[2].append(w[:, None] * temp * (torch.exp(z - lse[:, None]) - t))
    return [torch.cat(x) for x in out if x]


def _exact_attention(s, case):
    heads, kv, dim = case["heads"], case["kv"], case["dim"]
    outs = [torch.zeros(x.shape, dtype=torch.float64, device=DEV) for x in
            ([s["out"], s["lse"]] if case["kind"] == "attend" else [s["q"], s["k"], s["v"]])]
    q0 = k0 = 0
    for n, m in zip(_lens(case["lens_q"]), _lens(case["lens_k"])):
        rows, keys = slice(q0, q0 + n), slice(k0, k0 + m)
        q0, k0 = q0 + n, k0 + m
        gap = torch.arange(m, device=DEV)[None, :] - (torch.arange(n, device=DEV)[:, None] + (m - n))
        hidden = torch.zeros(n, m, dtype=torch.bool, device=DEV)
        if case["causal"]:
            hidden |= gap > 0
        if case["window"]:
            hidden |= gap.abs() >= case["window"]
        blind = hidden.all(1)
        for h in range(heads):
            c, e = slice(h * dim, (h + 1) * dim), h * kv // heads
            e = slice(e * dim, (e + 1) * dim)
            q, k, v = s["q"][rows, c].double(), s["k"][keys, e].double(), s["v"][keys, e].double()
            x = (torch.mm(q, k.t().contiguous()) * s["scale"]).masked_fill(hidden, -math.inf)
            if case["kind"] == "attend":
                lse = torch.logsumexp(x, 1)
                p = torch.exp(x - lse[:, None].masked_fill(blind[:, None], 0.0))
                outs[0][rows, c], outs[1][rows, h] = torch.mm(p, v), lse
                continue
            p = torch.exp(x - s["lse"][rows, h].double()[:, None].masked_fill(blind[:, None], 0.0))
            do, o = s["dout"][rows, c].double(), s["out"][rows, c].double()
            ds = p * (torch.mm(do, v.t().contiguous()) - (do * o).sum(1, keepdim=True)) * s["scale"]
            outs[0][rows, c] = torch.mm(ds, k)
            outs[1][keys, e] += torch.mm(ds.t().contiguous(), q)
            outs[2][keys, e] += torch.mm(p.t().contiguous(), do)
    return outs
