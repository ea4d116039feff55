"""The work that the operators which complete a token model are judged by: layer norm, linear attention by the gated delta rule,
and the verification of drafted tokens against the target's probabilities.

Every case is one call, or one forward and backward pair, that a program with a ``LAPLEX^(r)`` vocabulary head makes around that
head: while it reads prompts, writes tokens, checks drafted ones, or trains.  ``run`` computes it in plain torch operations where
``own`` is false, and through this library's entry points where it is true.
"""
from __future__ import annotations

import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


# --- the cases -------------------------------------------------------------------------------------------------------

def _norm(name, rows, width, dtype="bf16", step="forward", affine=True):
    """``rows`` rows of ``width`` numbers, with a weight and a bias or (not ``affine``) without."""
    return dict(name=name, op="norm", rows=rows, width=width, dtype=dtype, step=step, affine=affine)


def _delta(name, sequences, tokens, heads, key_heads, dk, dv, dtype="bf16", step="forward", packed=False, continues=False, part=False):
    """``tokens`` over all sequences, of equal lengths, or (``packed``) cut at random places, empty sequences among them; ``heads`` of
    values, ``key_heads`` of queries and keys; ``continues``: the sequences begin from states that earlier calls have left; ``part``:
    only so many of a sequence's tokens are read as a device array says."""
    return dict(name=name, op="delta", sequences=sequences, tokens=tokens, heads=heads, key_heads=key_heads, dk=dk, dv=dv, dtype=dtype,
                step=step, packed=packed, continues=continues, part=part)


def _verify(name, rows, sequences, columns, dtype="f32", drafts="logits", packed=False, banned=False, tau=1.0, near=0.5):
    """``rows`` logits (the vocabulary) for each of ``columns`` tokens of all sequences: as many as were drafted and one more for each
    sequence.  ``drafts``: "logits" (drawn from a smaller model's logits, which differ from the target's by ``near``), "sure" (looked
    up: they have no probabilities) or "greedy" (looked up, and compared with the likeliest token)."""
    return dict(name=name, op="verify", rows=rows, sequences=sequences, columns=columns, dtype=dtype, drafts=drafts, packed=packed,
                banned=banned, tau=tau, near=near)


def listed():
    return [
        # one token for each of 64 running sequences: what a call costs
        _norm("norm_tokens", 64, 4096),
        # a training step's norm before a projection
        _norm("norm_train", 32768, 4096, step="train"),
        # a training step's norm of queries and keys: 16384 tokens of 32 heads
        _norm("norm_heads_train", 16384 * 32, 128, step="train"),
        # the next token of one sequence
        _delta("delta_step_one", 1, 1, 16, 8, 128, 128, step="token"),
        # 256 sequences of which five tokens each were drafted and some accepted: these are read into the states
        _delta("delta_accepted", 256, 256 * 5, 16, 8, 128, 128, continues=True, part=True),
        # four prompts of ordinary length
        _delta("delta_prompts", 4, 4 * 2048, 16, 16, 128, 128),
        # one long document, read on from a state
        _delta("delta_long_prompt", 1, 65536, 8, 8, 128, 128, continues=True),
        # a training step, two heads of values to a head of keys
        _delta("delta_train", 8, 8 * 4096, 16, 8, 128, 128, step="train"),
        # a training step on documents of all lengths, packed, in fp32, with heads of odd sizes
        _delta("delta_train_packed", 24, 30011, 6, 3, 96, 80, dtype="f32", step="train", packed=True, continues=True),
        # four drafted tokens of one sequence, over the vocabulary head's 32000 rows
        _verify("verify_one", 32000, 1, 5),
        # four drafted tokens for each of 200 sequences on average; a mask has banned part of the vocabulary
        _verify("verify_serve", 32000, 200, 1001, packed=True, banned=True, tau=0.8),
        # tokens looked up in the text so far, eight for each of 64 sequences, a larger vocabulary of odd size
        _verify("verify_lookup", 60001, 64, 64 * 9, dtype="bf16", drafts="sure"),
    ]


def _log(rng, lo, hi):
    """A whole number from lo to hi, even over the logarithm; odd as often as even."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["norm", "norm", "delta", "delta", "delta", "token", "verify", "verify"])
    dtype = rng.choice(["f32", "bf16"])
    if kind == "norm":
        width = rng.choice([64, 80, 128, 256, 1000, 2048, 4096, _log(rng, 8, 16384), _log(rng, 8, 16384)])
        c = _norm("", _log(rng, 1, max(1, min(1 << 19, (1 << 26) // width))), width, dtype, rng.choice(["forward", "train"]), rng.random() < 0.8)
    elif kind == "delta":
        dk = rng.choice([32, 64, 64, 80, 96, 128, 128, 192, 256, rng.randint(1, 160)])
        dv = dk if rng.random() < 0.5 else rng.choice([32, 64, 96, 128, 160, 256, rng.randint(1, 160)])
        heads = rng.choice([1, 2, 3, 4, 6, 8, 12, 16])
        key_heads = rng.choice([d for d in (1, 2, 3, 4, 6, 8, 12, 16) if heads % d == 0 and heads // d <= 4])
        step = rng.choice(["forward", "train"])
        most = min(65536, (1 << 24) // (heads * max(dk, dv)) * (1 if dtype == "f32" else 2))
        sequences = _log(rng, 1, 64)
        if rng.random() < 0.5:
            c = _delta("", sequences, _log(rng, sequences, max(sequences, most)), heads, key_heads, dk, dv, dtype, step, True, rng.random() < 0.5,
                       rng.random() < 0.2)
        else:
            c = _delta("", sequences, sequences * _log(rng, 1, max(1, most // sequences)), heads, key_heads, dk, dv, dtype, step, False,
                       rng.random() < 0.5, rng.random() < 0.2)
    elif kind == "token":
        dk = rng.choice([32, 64, 80, 128, 128, 192, 256, rng.randint(1, 160)])
        dv = dk if rng.random() < 0.7 else rng.choice([64, 128, 256, rng.randint(1, 160)])
        heads = rng.choice([1, 2, 3, 6, 8, 12, 16, 32])
        sequences = _log(rng, 1, max(1, min(512, (1 << 26) // (heads * dk * dv))))
        c = _delta("", sequences, sequences, heads, heads if heads % 2 or rng.random() < 0.5 else heads // 2, dk, dv, dtype, "token")
    else:
        rows = _log(rng, 10, 131072)
        columns = _log(rng, 2, max(2, min(2048, (1 << 25) // rows)))
        each = rng.randint(1, min(9, columns))
        packed = rng.random() < 0.5
        sequences = max(1, columns // each)
        c = _verify("", rows, sequences, columns if packed else sequences * each, dtype, rng.choice(["logits", "logits", "sure", "greedy"]),
                    packed, rows >= 100 and rng.random() < 0.4, rng.choice([1.0, 1.0, 0.7, 1.3]), rng.choice([0.1, 0.5, 2.0]))
    del c["name"]
    return c


# --- inputs ----------------------------------------------------------------------------------------------------------

_EPS = 1e-5


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    uniform = lambda *shape, **kw: torch.rand(*shape, generator=gen, device="cuda", **kw)
    whole = lambda hi, *shape: torch.randint(0, hi, shape, generator=gen, device="cuda")
    new = lambda *shape, **kw: torch.empty(*shape, device="cuda", **kw)
    real = _TYPES[case["dtype"]]
    s = dict(case)
    if case["op"] == "norm":
        n, w = case["rows"], case["width"]
        # activations: rows of different sizes and means, some columns larger than the others
        s["x"] = (normal(n, w) * (0.5 + uniform(w)) * (0.5 + 2.0 * uniform(n, 1)) + normal(n, 1)).to(real)
        s.update(weight=1.0 + 0.2 * normal(w) if case["affine"] else None, bias=0.1 * normal(w) if case["affine"] else None,
                 y=new(n, w, dtype=real), mean=new(n), rstd=new(n))
        if case["step"] == "train":
            s.update(gy=normal(n, w).to(real), gx=new(n, w, dtype=real), ws=None)
            if case["affine"]:
                s.update(gweight=new(w), gbias=new(w))
    elif case["op"] == "delta":
        n, h, kh, dk, dv, b = (case[v] for v in ("tokens", "heads", "key_heads", "dk", "dv", "sequences"))
        split = lambda m: dict(zip(("q", "k", "v"), (m[:, :kh * dk].unflatten(1, (kh, dk)), m[:, kh * dk:2 * kh * dk].unflatten(1, (kh, dk)),
                                                     m[:, 2 * kh * dk:].unflatten(1, (h, dv)))))
        unit = lambda x: x / x.square().sum(-1, keepdim=True).sqrt()
        m = new(n, 2 * kh * dk + h * dv, dtype=real)                      # parts of one matrix, read where they lie
        s.update(split(m))
        s["q"].copy_(unit(normal(n, kh, dk)))
        s["k"].copy_(unit(normal(n, kh, dk)))
        s["v"].copy_(normal(n, h, dv))
        # decays from 0.999 to 0.4 a token, weights of a token anywhere between 0 and 1
        s.update(rates=torch.exp(-7.0 + 7.0 * uniform(n, h)), beta=torch.sigmoid(normal(n, h)), scale=dk ** -0.5, starts=None, lengths=None,
                 longest=n // b)
        s["y"] = torch.zeros(n, h, dv, device="cuda", dtype=real)
        if case["packed"]:
            cuts = torch.sort(whole(n + 1, b - 1)).values
            s["starts"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), n)])
            s["longest"] = int((s["starts"][1:] - s["starts"][:-1]).max())
        if case["part"]:
            s["lengths"] = whole(s["longest"] + 1, b)                     # beyond a sequence's end: all of it
        if case["continues"] or case["step"] == "token":
            s["state"] = normal(b, h, dk, dv)
        if case["step"] != "token":
            s.update(state_out=new(b, h, dk, dv), ws=None, ws_for=(n, b, h, kh, dk, dv))
        if case["step"] == "train":
            s["gy"] = normal(n, h, dv).to(real)
            s.update({"g" + v: t for v, t in split(torch.zeros_like(m)).items()})
            s.update(grates=torch.zeros(n, h, device="cuda"), gbeta=torch.zeros(n, h, device="cuda"))
            if case["continues"]:
                s.update(gstate_out=normal(b, h, dk, dv), gstate=new(b, h, dk, dv))
    else:
        k, b, t = case["rows"], case["sequences"], case["columns"]
        s["drafts_are"] = case["drafts"]
        z = 4.0 * normal(k, t)                                            # the smaller model's logits, and the target's
        y = z + case["near"] * normal(k, t)
        if case["banned"]:
            y.masked_fill_(uniform(k, t) < 0.05, -math.inf)
        s.update(y=y.to(real), z=z.to(real) if case["drafts"] == "logits" else None, starts=None, ws=None, draft_tau=1.0)
        # drafts drawn from the smaller model: the largest of its logits with noise of a Gumbel law
        if case["drafts"] == "greedy":
            s["drafts"] = s["y"].argmax(0)
            s["drafts"] = torch.where(uniform(t) < 0.3, whole(k, t), s["drafts"])
        else:
            smaller = s["z"].float() if s["z"] is not None else y
            s["drafts"] = (smaller - torch.log(-torch.log(uniform(k, t).clamp(min=1e-30)).clamp(min=1e-30))).argmax(0)
        s["drafts"][uniform(t) < 0.02] = -1                               # nothing was drafted from here on
        if case["packed"]:
            cuts = torch.sort(whole(t + 1, b - 1)).values
            s["starts"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), t)])
        s.update(chances=uniform(t, dtype=torch.float64), next_chances=uniform(b, dtype=torch.float64), accepted=new(b, dtype=torch.int64),
                 following=new(b, dtype=torch.int64), logp=new(t), following_logp=new(b))
        s["most"] = int((s["starts"][1:] - s["starts"][:-1]).max()) if case["packed"] else t // b
    return s


# --- the plain forms -------------------------------------------------------------------------------------------------

def _plain_norm(s):
    x, real = s["x"].float(), s["x"].dtype
    mean = x.mean(1)
    centred = x - mean[:, None]
    rstd = torch.rsqrt(centred.square().mean(1) + _EPS)
    hat = centred * rstd[:, None]
    affine = s["weight"] is not None
    out = {"y": (hat * s["weight"] + s["bias"] if affine else hat).to(real), "mean": mean, "rstd": rstd}
    if s["step"] == "train":
        gy = s["gy"].float()
        g = gy * s["weight"] if affine else gy
        out["gx"] = ((g - g.mean(1, keepdim=True) - hat * (g * hat).mean(1, keepdim=True)) * rstd[:, None]).to(real)
        if affine:
            out.update(gweight=(gy * hat).sum(0), gbias=gy.sum(0))
    return out


_CHUNK = 64


def _inverse(a):
    """(1 + a)^-1 of strictly lower triangular matrices: blocks of 1, 2, 4, ... on the diagonal are joined by what lies below them."""
    n = a.shape[-1]
    at = torch.arange(n, device=a.device)
    t = torch.eye(n, device=a.device).expand_as(a)
    size = 1
    while size < n:
        block = at // size
        below = (block[:, None] == block + 1) & (block % 2 == 0)
        t = t - t @ (a * below) @ t
        size *= 2
    return t


class _Chunks:
    """The delta rule on (sequences, heads, chunks, tokens of a chunk, .): inside chunks by triangular matrices, and from chunk to
    chunk by state <- m state + p."""

    def __init__(self, q, k, v, rates, beta):
        turn = lambda x: x.transpose(-1, -2).contiguous()
        self.q, self.k, self.v, self.beta = q, k, v, beta[..., None]
        g = torch.cumsum(-rates.double(), -1)                              # differences of far sums: in 64 bits
        n = g.shape[-1]
        at = torch.arange(n, device=q.device)
        apart = torch.where(at[:, None] >= at, g[..., :, None] - g[..., None, :], -math.inf)
        self.apart = torch.exp(apart).float()
        self.ahead = torch.exp(g).float()[..., None]
        self.behind = torch.exp(g[..., -1:] - g).float()[..., None]
        self.whole = self.ahead[..., -1:, :]
        self.kk = k @ turn(k)
        self.below = (at[:, None] > at).float()
        self.a = self.beta * self.apart * self.kk * self.below
        self.t = _inverse(self.a)
        self.w = self.t @ (self.beta * self.ahead * k)
        self.p = self.apart * (q @ turn(k))
        self.late = self.behind * k
        self.m = self.whole * torch.eye(k.shape[-1], device=k.device) - turn(self.late) @ self.w
        self.turn = turn

    def forward(self, state):
        """(results, state of each chunk's beginning, the tokens' corrections, last state)"""
        u = self.t @ (self.beta * self.v)
        add = self.turn(self.late) @ u
        states = torch.empty(add.shape[:2] + (add.shape[2] + 1,) + add.shape[3:], device=add.device)
        states[:, :, 0] = 0.0 if state is None else state
        for c in range(add.shape[2]):
            states[:, :, c + 1] = self.m[:, :, c] @ states[:, :, c] + add[:, :, c]
        first = states[:, :, :-1]
        u = u - self.w @ first
        return self.ahead * (self.q @ first) + self.p @ u, first, u, states[:, :, -1]

    def backward(self, gy, first, u, glast):
        turn = self.turn
        back = turn(self.p) @ gy
        add = turn(self.ahead * self.q) @ gy - turn(self.w) @ back
        states = torch.empty(add.shape[:2] + (add.shape[2] + 1,) + add.shape[3:], device=add.device)
        states[:, :, -1] = 0.0 if glast is None else glast
        m = turn(self.m)
        for c in range(add.shape[2] - 1, -1, -1):
            states[:, :, c] = m[:, :, c] @ states[:, :, c + 1] + add[:, :, c]
        g = states[:, :, 1:].contiguous()
        gr = turn(self.t) @ (back + self.late @ g)
        ga = -(gr @ turn(u)) * self.below
        gp = gy @ turn(u)
        n, m = gp * self.apart, ga * self.apart
        dots = lambda x, y: (x * y).sum(-1)
        from_state = gr @ turn(first)
        ahead, behind, beta = self.ahead[..., 0], self.behind[..., 0], self.beta[..., 0]
        into_state = u @ turn(g)
        q_state = self.ahead * (gy @ turn(first))
        gq = n @ self.k + q_state
        both = self.beta * m
        gk = turn(n) @ self.q + both @ self.k + turn(both) @ self.k - self.beta * self.ahead * from_state + self.behind * into_state
        taken = ahead * dots(self.k, from_state)
        gbeta = dots(gr, self.v) - taken + (m * self.kk).sum(-1)
        late = behind * dots(self.k, into_state)
        in_a, in_p = ga * self.a, gp * self.p
        gg = in_p.sum(-1) - in_p.sum(-2) + in_a.sum(-1) - in_a.sum(-2) - beta * taken - late + dots(self.q, q_state)
        gg[..., -1] += late.sum(-1) + self.whole[..., 0, 0] * (first * g).sum((-1, -2))
        grates = -gg.flip(-1).cumsum(-1).flip(-1)
        return gq, gk, self.beta * gr, grates, gbeta, states[:, :, 0]


def _rows(s):
    """(row of every token of every sequence, whether it is read): sequences one beside the other, in whole chunks."""
    b, dev = s["sequences"], s["q"].device
    starts = s["starts"] if s["starts"] is not None else torch.arange(b + 1, device=dev) * s["longest"]
    lengths = starts[1:] - starts[:-1]
    if s["lengths"] is not None:
        lengths = torch.minimum(lengths, s["lengths"])
    at = torch.arange(max(1, -(-s["longest"] // _CHUNK)) * _CHUNK, device=dev)
    return starts[:-1, None] + at, at < lengths[:, None]


def _plain_delta(s):
    row, there = _rows(s)
    some = row.clamp(max=s["tokens"] - 1)
    group = s["heads"] // s["key_heads"]
    real, scale = s["q"].dtype, s["scale"]

    def spread(x):                                                         # (sequences, heads, chunks, tokens, .)
        x = x[some].float() * there.reshape(there.shape + (1,) * (x.dim() - 1))
        x = x.transpose(1, 2)
        if x.shape[1] != s["heads"]:
            x = x.repeat_interleave(group, 1)
        return x.unflatten(2, (-1, _CHUNK)).contiguous()

    def gather(x, like):
        out = torch.zeros_like(like)
        x = x.flatten(2, 3)
        if x.shape[1] != like.shape[1]:
            x = x.unflatten(1, (-1, group)).sum(2)
        out[row[there]] = x.transpose(1, 2)[there].to(out.dtype)
        return out

    c = _Chunks(scale * spread(s["q"]), spread(s["k"]), spread(s["v"]), spread(s["rates"]), spread(s["beta"]))
    y, first, u, last = c.forward(s.get("state"))
    out = {"y": gather(y, s["y"]), "state": last}
    if s["step"] == "train":
        gq, gk, gv, grates, gbeta, gstate = c.backward(spread(s["gy"]), first, u, s.get("gstate_out"))
        out.update(gq=gather(scale * gq, s["gq"]), gk=gather(gk, s["gk"]), gv=gather(gv, s["gv"]), grates=gather(grates, s["grates"]),
                   gbeta=gather(gbeta, s["gbeta"]))
        if "gstate" in s:
            out["gstate"] = gstate
    return out


def _plain_token(s):
    group = s["heads"] // s["key_heads"]
    q, k, v = s["q"].float().repeat_interleave(group, 1), s["k"].float().repeat_interleave(group, 1), s["v"].float()
    state = s["state"].mul_(torch.exp(-s["rates"])[..., None, None])
    u = s["beta"][..., None] * (v - (k[..., None] * state).sum(-2))
    state.add_(k[..., None] * u[..., None, :])
    return {"y": (s["scale"] * (q[..., None] * state).sum(-2)).to(s["q"].dtype), "state": state}


def _probabilities(y, tau):
    z = y.double() * tau
    e = torch.exp(z - z.max(0).values)
    return e / e.sum(0)


def _plain_verify(s):
    """In 64 bits: a comparison of two probabilities, or of a chance and a running sum, turns on their last ones."""
    t, b, k = s["columns"], s["sequences"], s["rows"]
    dev = s["y"].device
    tau, draft_tau = (float(torch.tensor(s[v], dtype=torch.float32)) for v in ("tau", "draft_tau"))
    starts = s["starts"] if s["starts"] is not None else torch.arange(b + 1, device=dev) * (t // b)
    ends = starts[1:] - 1                                                  # a sequence's last column has no draft to judge
    at = starts[:-1, None] + torch.arange(s["most"], device=dev)
    drafts = s["drafts"]
    given = (drafts >= 0) & (drafts < k)
    x = torch.where(given, drafts, 0)[None]
    p = _probabilities(s["y"], tau)
    if s["drafts_are"] == "greedy":
        best = torch.where(s["y"] == s["y"].max(0).values, torch.arange(k, device=dev)[:, None], k).min(0).values
        kept = given & (drafts == best)
    else:
        q = _probabilities(s["z"], draft_tau) if s["z"] is not None else None
        kept = given & (s["chances"] * (1.0 if q is None else q.gather(0, x)[0]) < p.gather(0, x)[0])
    there = at < ends[:, None]
    going = there & kept[at.clamp(max=t - 1)]
    accepted = going.long().cumprod(1).sum(1)
    column = (starts[:-1] + accepted).clamp(max=t - 1)
    empty = ends < starts[:-1]
    if s["drafts_are"] == "greedy":
        following = best[column]
    else:
        w = p[:, column]
        judged = (column < ends) & given[column]                           # refused: what the drafts had too much of is taken out
        if q is None:
            w = w.scatter(0, x[:, column], torch.where(judged, 0.0, w.gather(0, x[:, column])[0])[None])
        else:
            left = (w - q[:, column]).clamp(min=0.0)
            w = torch.where(judged & (left.sum(0) > 0.0), left, w)
        run_ = w.cumsum(0)
        past = (run_ > s["next_chances"] * run_[-1]) & (w > 0.0)
        following = torch.where(past, torch.arange(k, device=dev)[:, None], k).min(0).values
    judged = torch.zeros(t, dtype=torch.bool, device=dev)
    judged[at[there]] = True
    logp = torch.where(judged & given, torch.log(p.gather(0, x)[0]), 0.0)
    following_logp = torch.where(empty, 0.0, torch.log(p[following.clamp(max=k - 1), column]))
    return {"accepted": torch.where(empty, 0, accepted), "next": torch.where(empty, -1, following), "logp": logp.float(),
            "next_logp": following_logp.float()}


# --- one pass --------------------------------------------------------------------------------------------------------

def _workspace(s, size):
    """A program keeps its workspace from call to call."""
    if s["ws"] is None:
        s["ws"] = torch.empty(size(), dtype=torch.uint8, device="cuda")
    return s["ws"]


def _own(s):
    from paper_2605_24584_amd import binding as B
    if s["op"] == "norm":
        B.laplex_layer_norm(s["x"], s["weight"], s["bias"], s["y"], s["mean"], s["rstd"], _EPS)
        out = {v: s[v] for v in ("y", "mean", "rstd")}
        if s["step"] == "train":
            ws = _workspace(s, lambda: B.laplex_layer_norm_workspace_bytes(s["rows"], s["width"]))
            B.laplex_layer_norm_backward(s["x"], s["gy"], s["weight"], s["mean"], s["rstd"], s["gx"], s.get("gweight"), s.get("gbias"), ws)
            out.update({v: s[v] for v in ("gx", "gweight", "gbias") if v in s})
        return out
    if s["op"] == "verify":
        ws = _workspace(s, lambda: B.laplex_verify_workspace_bytes(s["rows"], s["columns"], s["sequences"]))
        B.laplex_verify_drafts(s["y"], s["z"], s["drafts"], s["chances"], s["next_chances"], s["accepted"], s["following"], ws, s["logp"],
                               s["following_logp"], s["tau"], s["draft_tau"], s["sequences"], s["starts"], B.LAPLEX_VERIFY_GREEDY if s["drafts_are"] == "greedy" else 0)
        return {"accepted": s["accepted"], "next": s["following"], "logp": s["logp"], "next_logp": s["following_logp"]}
    if s["step"] == "token":
        B.laplex_delta_attention_step(s["q"], s["k"], s["v"], s["rates"], s["beta"], s["state"], s["y"], s["scale"])
        return {"y": s["y"], "state": s["state"]}
    train = s["step"] == "train"
    ws = _workspace(s, lambda: B.laplex_delta_attention_workspace_bytes(s["q"].dtype, *s["ws_for"], train))
    keep = B.LAPLEX_SAVE_SCANS if train else 0
    B.laplex_delta_attention(s["q"], s["k"], s["v"], s["rates"], s["beta"], s["y"], ws, s["scale"], s["sequences"], s["starts"], s["lengths"],
                             s.get("state"), s["state_out"], keep)
    out = {"y": s["y"], "state": s["state_out"]}
    if train:
        B.laplex_delta_attention_backward(s["q"], s["k"], s["v"], s["rates"], s["beta"], s["gy"], s["gq"], s["gk"], s["gv"], s["grates"],
                                          s["gbeta"], ws, s["scale"], s["sequences"], s["starts"], s["lengths"], s.get("state"),
                                          s.get("gstate_out"), s.get("gstate"), keep)
        out.update({v: s[v] for v in ("gq", "gk", "gv", "grates", "gbeta", "gstate") if v in s})
    return out


def run(state):
    if own:
        return _own(state)
    if state["op"] == "norm":
        return _plain_norm(state)
    if state["op"] == "verify":
        return _plain_verify(state)
    return _plain_token(state) if state["step"] == "token" else _plain_delta(state)


# --- the definitions in 64 bits ----------------------------------------------------------------------------------------

def _exact_norm(s):
    x, w = s["x"].double(), s["width"]
    mean = x.sum(1) / w
    var = (x - mean[:, None]).square().sum(1) / w
    rstd = 1.0 / (var + _EPS).sqrt()
    weight = torch.ones(w, device=x.device, dtype=torch.float64) if s["weight"] is None else s["weight"].double()
    hat = (x - mean[:, None]) / (var + _EPS).sqrt()[:, None]
    out = {"y": hat * weight + (0.0 if s["bias"] is None else s["bias"].double()), "mean": mean, "rstd": rstd}
    if s["step"] == "train":
        gy = s["gy"].double()
        ghat = gy * weight
        # the row's Jacobian, (1 - 1 1^T / w - hat hat^T / w) / std
        out["gx"] = rstd[:, None] * (ghat - (ghat.sum(1, keepdim=True) + hat * (ghat * hat).sum(1, keepdim=True)) / w)
        if s["weight"] is not None:
            out.update(gweight=torch.einsum("nw,nw->w", gy, hat), gbias=gy.sum(0))
    return out


_KEPT = 64


def _exact_delta(s):
    """Token after token by the definition, all sequences and heads side by side; backwards from states that are kept every so often."""
    b, h, kh, dk, dv, n = (s[v] for v in ("sequences", "heads", "key_heads", "dk", "dv", "longest"))
    dev, group, train = s["q"].device, h // kh, s["step"] == "train"
    starts = s["starts"] if s["starts"] is not None else torch.arange(b + 1, device=dev) * n
    at = torch.arange(max(n, 1), device=dev)
    last = torch.minimum(starts[1:], starts[:-1] + s["lengths"]) if s["lengths"] is not None else starts[1:]
    row = (starts[:-1] + at[:, None]).clamp(max=s["tokens"] - 1)
    there = starts[:-1] + at[:, None] < last                              # (tokens, sequences)

    def lay(x, wide):                                                     # (tokens, sequences * heads, .)
        x = x.double()[row] * there.reshape(there.shape + (1,) * (x.dim() - 1))
        if wide:
            x = x.repeat_interleave(group, 2)
        return x.flatten(1, 2)

    q, k, v = lay(s["q"], True) * s["scale"], lay(s["k"], True), lay(s["v"], False)
    decay, beta = torch.exp(-lay(s["rates"], False)), lay(s["beta"], False)
    state = s["state"].double().flatten(0, 1).clone() if "state" in s else torch.zeros(b * h, dk, dv, dtype=torch.float64, device=dev)
    y = torch.zeros_like(v)

    def token(t, state):
        before = decay[t][:, None, None] * state
        miss = v[t] - torch.bmm(k[t][:, None], before)[:, 0]
        return before, miss, torch.baddbmm(before, k[t][:, :, None], (beta[t][:, None] * miss)[:, None])

    kept = []
    for t in range(n):
        if train and t % _KEPT == 0:
            kept.append(state.clone())
        _, _, state = token(t, state)
        y[t] = torch.bmm(q[t][:, None], state)[:, 0]

    def lie(x, like, wide=False):
        x = x.unflatten(1, (b, h))
        if wide:
            x = x.unflatten(2, (kh, group)).sum(3)
        out = torch.zeros(like.shape, dtype=torch.float64, device=dev)
        out[row[there]] = x[there[:len(x)]]
        return out

    out = {"y": lie(y, s["y"]), "state": state.unflatten(0, (b, h))}
    if not train:
        return out
    gy = lay(s["gy"], False)
    gq, gk, gv, gr, gb = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v), torch.zeros_like(beta), torch.zeros_like(beta)
    g = s["gstate_out"].double().flatten(0, 1).clone() if "gstate_out" in s else torch.zeros_like(state)
    for lo in range((n - 1) // _KEPT * _KEPT, -1, -_KEPT):
        steps, state = [], kept.pop()
        for t in range(lo, min(n, lo + _KEPT)):
            steps.append((t,) + token(t, state))
            state = steps[-1][-1]
        for t, before, miss, after in reversed(steps):
            gq[t] = torch.bmm(after, gy[t][:, :, None])[..., 0]
            g = torch.baddbmm(g, q[t][:, :, None], gy[t][:, None])
            gu = torch.bmm(k[t][:, None], g)[:, 0]
            gb[t] = (gu * miss).sum(-1)
            gv[t] = beta[t][:, None] * gu
            gk[t] = torch.bmm(g, (beta[t][:, None] * miss)[:, :, None])[..., 0] - torch.bmm(before, gv[t][:, :, None])[..., 0]
            g = torch.baddbmm(g, k[t][:, :, None], gv[t][:, None], alpha=-1.0)
            gr[t] = -(g * before).sum((1, 2))
            g = decay[t][:, None, None] * g
    out.update(gq=lie(gq * s["scale"], s["gq"], True), gk=lie(gk, s["gk"], True), gv=lie(gv, s["gv"]), grates=lie(gr, s["grates"]),
               gbeta=lie(gb, s["gbeta"]))
    if "gstate" in s:
        out["gstate"] = g.unflatten(0, (b, h))
    return out


def _exact_token(s):
    group = s["heads"] // s["key_heads"]
    q, k = (s[v].double().repeat_interleave(group, 1) for v in "qk")
    before = torch.exp(-s["rates"].double())[..., None, None] * s["state"].double()
    miss = s["v"].double() - torch.einsum("bhk,bhkv->bhv", k, before)
    last = before + torch.einsum("bhk,bh,bhv->bhkv", k, s["beta"].double(), miss)
    return {"y": s["scale"] * torch.einsum("bhk,bhkv->bhv", q, last), "state": last}


def _exact_verify(s):
    """One sequence after the other, one draft after the other."""
    b, k, dev = s["sequences"], s["rows"], s["y"].device
    starts = s["starts"].tolist() if s["starts"] is not None else [i * (s["columns"] // b) for i in range(b + 1)]
    tau = torch.tensor(s["tau"], dtype=torch.float32, device=dev).double()
    logp, next_logp = torch.zeros(s["columns"], dtype=torch.float64, device=dev), torch.zeros(b, dtype=torch.float64, device=dev)
    accepted, following = torch.zeros(b, dtype=torch.int64, device=dev), torch.full((b,), -1, device=dev)
    drafts, chances, next_chances = s["drafts"].tolist(), s["chances"].tolist(), s["next_chances"].tolist()
    for i in range(b):
        going = True
        for c in range(starts[i], starts[i + 1]):
            of = torch.log_softmax(s["y"][:, c].double() * tau, 0)
            x = drafts[c] if c + 1 < starts[i + 1] and 0 <= drafts[c] < k else None
            if x is not None:
                logp[c] = of[x]
            if not going:
                continue
            p, q = of.exp(), None
            if s["drafts_are"] == "greedy":
                best = int((s["y"][:, c] == s["y"][:, c].max()).nonzero()[0])
                if x == best:
                    accepted[i] += 1
                    continue
                following[i], next_logp[i], going = best, of[best], False
                continue
            if x is not None and s["z"] is not None:
                q = torch.softmax(s["z"][:, c].double() * s["draft_tau"], 0)
            elif x is not None:
                q = torch.zeros_like(p)
                q[x] = 1.0
            if x is not None and chances[c] * float(q[x]) < float(p[x]):
                accepted[i] += 1
                continue
            left = p if q is None else (p - q).clamp(min=0.0)
            edges = torch.cumsum(left if float(left.sum()) > 0.0 else p, 0)
            at = int(torch.searchsorted(edges, edges[-1:] * next_chances[i], right=True))
            following[i], next_logp[i], going = at, of[at], False
    return {"accepted": accepted, "next": following, "logp": logp, "next_logp": next_logp}


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "verify":
        return _exact_verify(s)
    if case["op"] == "norm":
        return _exact_norm(s)
    return _exact_token(s) if case["step"] == "token" else _exact_delta(s)


# --- what a pass cannot do without -------------------------------------------------------------------------------------

def work(case):
    """Each input read once and each output written once, forward and backward apart (the loss lies between them).  Delta rule: the
    recurrence's multiply-adds, dk * dv each for a token's product with the state, for the state's change and for the result; backwards as
    many again for the states, and four for the gradients.  Verification: both matrices once; an exponential counts as one operation."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "norm":
        n, w = case["rows"], case["width"]
        moved, flops = 2 * e * n * w + 8 * n + 8 * w, 8.0 * n * w
        if case["step"] == "train":
            moved, flops = moved + 3 * e * n * w + 8 * n + 12 * w, flops + 14.0 * n * w
        return {"bytes": moved, "flops": flops}
    if case["op"] == "verify":
        k, t, b = case["rows"], case["columns"], case["sequences"]
        both = 2 if case["drafts"] == "logits" else 1
        return {"bytes": both * e * k * t + 20 * t + 28 * b, "flops": both * 3.0 * k * t}
    n, h, kh, dk, dv, b = (case[v] for v in ("tokens", "heads", "key_heads", "dk", "dv", "sequences"))
    rows, small, state = e * n * (2 * kh * dk + 2 * h * dv), 8 * n * h, 4 * b * h * dk * dv
    begins = 1 if case["continues"] or case["step"] == "token" else 0
    moved, flops = rows + small + state * (1 + begins), 6.0 * n * h * dk * dv
    if case["step"] == "train":
        moved += e * n * (4 * kh * dk + 3 * h * dv) + 2 * small + state * 3 * begins
        flops += 14.0 * n * h * dk * dv
    return {"bytes": moved, "flops": flops}
