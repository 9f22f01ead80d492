"""Attention of a serving step, as measurable cases: the operators that make the
rows which an attention hook reads and writes.

Each case is one call as a serving program makes it for one layer.  `run` computes
the operators in plain torch operations in 32 bits, or, where `own` is set, through
the package's calls.

  norm_rope  norm of every query and key head with the position rotation; queries
             and keys are parts of one projection's output, so their rows are strided
  append     a step's keys and values into the pages of their requests, the keys
             rotated on the way or already rotated
  attend     the step's queries over the pages of their requests: one token each
             (decode), a few drafted ones, chunks of a prefill, or a mix

Head counts and widths are those of the served models' shapes (rows of 4096 and 8192
in heads of 128) and smaller ones; batches of 256 and 512 requests, chunks of up
to 8192 tokens and prompts of 128 to 1024 as in the synthetic workloads.
"""
import math
import random

import torch

own = False

DEV = "cuda"
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f32": 4, "e4m3": 1}
THETA = 500000.0
E4M3_MOST = 448.0


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # a decode step of 256 requests of an 8B-shaped model with normed heads
        dict(name="norm_rope_decode", kind="norm_rope", dtype="bf16", T=256, n_q=32, n_kv=8, hd=128,
             rot=128, pairs=False, norm=True, far=32768),
        # a full prefill chunk of a 70B-shaped model, rotation only
        dict(name="norm_rope_chunk", kind="norm_rope", dtype="bf16", T=8192, n_q=64, n_kv=8, hd=128,
             rot=128, pairs=False, norm=False, far=131072),
        # the smallest call: an fp32 toy of sixteen tokens, half of each head rotated
        # in neighbouring pairs
        dict(name="norm_rope_toy", kind="norm_rope", dtype="f32", T=16, n_q=8, n_kv=2, hd=64, rot=32,
             pairs=True, norm=True, far=512),
        # a decode step's keys and values, keys rotated on the way
        dict(name="append_decode", kind="append", dtype="bf16", cache="bf16", R=256, n_chunk=0, q_lo=1,
             q_hi=1, ctx_lo=0, ctx_hi=128, n_kv=8, hd=128, page=16, rot=128, pairs=False, mix=1),
        # a prefill chunk of sixteen prompts into 8-bit pages, keys normed and rotated before
        dict(name="append_chunk_e4m3", kind="append", dtype="bf16", cache="e4m3", R=16, n_chunk=16,
             q_lo=128, q_hi=1024, ctx_lo=0, ctx_hi=64, n_kv=8, hd=128, page=64, rot=0, pairs=False,
             mix=2),
        # one request decoding by itself: latency
        dict(name="attend_one", kind="attend", cache="bf16", R=1, n_chunk=0, q_lo=1, q_hi=1, ctx_lo=1023,
             ctx_hi=1023, n_q=32, n_kv=8, hd=128, page=16, window=0, mix=3),
        # a decode step of 256 requests with contexts from a few tokens to 8192
        dict(name="attend_decode", kind="attend", cache="bf16", R=256, n_chunk=0, q_lo=1, q_hi=1,
             ctx_lo=1, ctx_hi=8191, n_q=32, n_kv=8, hd=128, page=16, window=0, mix=4),
        # few requests with long contexts in 8-bit pages, 70B-shaped
        dict(name="attend_long_e4m3", kind="attend", cache="e4m3", R=24, n_chunk=0, q_lo=1, q_hi=1,
             ctx_lo=8192, ctx_hi=65536, n_q=64, n_kv=8, hd=128, page=64, window=0, mix=5),
        # five tokens a request to verify, in a model with a window
        dict(name="attend_drafts", kind="attend", cache="bf16", R=64, n_chunk=64, q_lo=5, q_hi=5,
             ctx_lo=100, ctx_hi=8000, n_q=32, n_kv=8, hd=128, page=32, window=4096, mix=6),
        # a continuous batch: a chunk of one prompt among decoding requests, heads of 64
        dict(name="attend_mixed", kind="attend", cache="bf16", R=96, n_chunk=1, q_lo=1001, q_hi=1001,
             ctx_lo=17, ctx_hi=4000, n_q=32, n_kv=8, hd=64, page=16, window=0, mix=7),
        # sixteen prompts of 128 to 1024 tokens prefilled together, 70B-shaped
        dict(name="attend_prompts", kind="attend", cache="bf16", R=16, n_chunk=16, q_lo=128, q_hi=1024,
             ctx_lo=0, ctx_hi=0, n_q=64, n_kv=8, hd=128, page=64, window=0, mix=8),
        # a chunk of a long prompt over what is cached of it: the largest
        dict(name="attend_chunk", kind="attend", cache="bf16", R=1, n_chunk=1, q_lo=4096, q_hi=4096,
             ctx_lo=28672, ctx_hi=28672, n_q=32, n_kv=8, hd=128, page=64, window=0, mix=9),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["norm_rope", "append", "attend", "attend", "attend"])
    mix = rng.randrange(1 << 20)
    n_kv = rng.choice([1, 2, 4, 8])
    hd = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    if kind == "norm_rope":
        hd = rng.choice([64, 128, 128, 256])
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]), T=_spread(rng, 16, 4096),
                    n_q=n_kv * rng.choice([1, 4, 7, 8]), n_kv=n_kv, hd=hd,
                    rot=rng.choice([hd, hd // 2]), pairs=rng.random() < 0.3, norm=rng.random() < 0.6,
                    far=_spread(rng, 100, 131072))
    if kind == "append":
        chunks = rng.random() < 0.5
        R = _spread(rng, 1, 16 if chunks else 512)
        return dict(kind=kind, dtype=rng.choice(["bf16", "bf16", "f32"]),
                    cache=rng.choice(["bf16", "e4m3"]), R=R, n_chunk=R if chunks else 0, q_lo=1,
                    q_hi=rng.randint(100, 1000) if chunks else 1, ctx_lo=0, ctx_hi=rng.randint(1, 256),
                    n_kv=n_kv, hd=hd, page=page, rot=rng.choice([0, hd, hd // 2]),
                    pairs=rng.random() < 0.3, mix=mix)
    form = rng.choice(["decode", "decode", "drafts", "mixed", "chunks"])
    d = dict(kind=kind, cache=rng.choice(["bf16", "bf16", "e4m3"]), R=1, n_chunk=0, q_lo=1, q_hi=1,
             ctx_lo=1, ctx_hi=1, n_q=n_kv * rng.choice([1, 4, 7, 8]), n_kv=n_kv, hd=hd, page=page,
             window=rng.choice([0, 0, 0, 1000, 4096]), mix=mix)
    if form == "decode":
        d["R"] = _spread(rng, 1, 256)
        d["ctx_hi"] = _spread(rng, 200, min(65536, 1 << 21) // max(1, d["R"] // 16))
    elif form == "drafts":
        d["R"] = d["n_chunk"] = _spread(rng, 1, 128)
        d["q_lo"], d["q_hi"] = 2, rng.randint(2, 8)
        d["ctx_hi"] = _spread(rng, 200, 8192)
    elif form == "mixed":
        d["R"], d["n_chunk"] = rng.randint(4, 128), rng.randint(1, 3)
        d["q_lo"], d["q_hi"] = 20, rng.randint(100, 1000)
        d["ctx_hi"] = _spread(rng, 200, 4096)
    else:
        d["R"] = d["n_chunk"] = rng.randint(1, 8)
        d["q_lo"], d["q_hi"] = 1, rng.randint(100, 2000)
        d["ctx_lo"], d["ctx_hi"] = 0, _spread(rng, 16, 4096)
    return d


def lengths(case):
    """New tokens and cached ones before them, of each request of the batch."""
    r = random.Random(case["mix"])
    n = [r.randint(case["q_lo"], case["q_hi"]) if i < case["n_chunk"] else 1 for i in range(case["R"])]
    ctx = [r.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["R"])]
    both = list(zip(n, ctx))
    r.shuffle(both)
    return [a for a, _ in both], [b for _, b in both]


def work(case):
    hd, n_kv = case["hd"], case["n_kv"]
    if case["kind"] == "norm_rope":
        rows = case["T"] * (case["n_q"] + n_kv)
        return {"bytes": 2 * rows * hd * SIZE[case["dtype"]] + 4 * case["T"], "flops": 10 * rows * hd}
    n, ctx = lengths(case)
    if case["kind"] == "append":
        rows = 2 * sum(n) * n_kv
        return {"bytes": rows * hd * (SIZE[case["dtype"]] + SIZE[case["cache"]]) + 8 * sum(n),
                "flops": 4 * rows * hd}
    keys = pairs = 0
    for a, c in zip(n, ctx):
        w = case["window"] or a + c
        pairs += sum(min(w, c + i + 1) for i in range(a))
        keys += min(a + c, w + a - 1)
    T = sum(n)
    return {"bytes": 2 * keys * n_kv * hd * SIZE[case["cache"]] + T * case["n_q"] * (4 * hd + 4),
            "flops": 4 * hd * case["n_q"] * pairs}


# ------------------------------------------------------------------ the inputs

def _frequencies(rot):
    return THETA ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)


def _normal(g, *shape, dtype=torch.float32):
    """Normal values with a few strong channels, as projections of a model's rows have."""
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
    x[..., 5] *= 4.0
    return x.to(dtype)


def _pages(case, n, ctx, g):
    """The cache's pages in no order, each request's table of them, and scales."""
    total, ps = [a + c for a, c in zip(n, ctx)], case["page"]
    count = [-(-t // ps) for t in total]
    order = list(range(sum(count) + 3))
    random.Random(case["mix"] + 1).shuffle(order)
    table, at = [], 0
    for c in count:
        table.append(order[at:at + c] + [-1] * (max(count) - c))
        at += c
    s = dict(table=torch.tensor(table, dtype=torch.int32, device=DEV), k_scale=None, v_scale=None)
    for name in ("k", "v"):
        x = _normal(g, len(order), case["n_kv"], ps, case["hd"], dtype=torch.bfloat16)
        if case["cache"] == "e4m3":
            s[name + "_scale"] = 0.02 + 0.02 * torch.rand(case["n_kv"], generator=g, device=DEV)
            x = (x.float() / s[name + "_scale"][:, None, None]).clamp(-E4M3_MOST, E4M3_MOST)
        s[name + "_pages"] = x.to(DT[case["cache"]])
    return s


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    s = dict(case=case)
    if case["kind"] == "norm_rope":
        dt, T, n_q, n_kv, hd = DT[case["dtype"]], case["T"], case["n_q"], case["n_kv"], case["hd"]
        row = _normal(g, T, n_q + 2 * n_kv, hd, dtype=dt)  # one projection's output
        s.update(q=row[:, :n_q], k=row[:, n_q:n_q + n_kv], eps=1e-6, q_w=None, k_w=None,
                 pos=torch.randint(0, case["far"], (T,), generator=g, device=DEV, dtype=torch.int32),
                 q_out=torch.zeros(T, n_q, hd, dtype=dt, device=DEV),
                 k_out=torch.zeros(T, n_kv, hd, dtype=dt, device=DEV))
        if case["norm"]:
            for name in ("q_w", "k_w"):
                s[name] = (1.0 + 0.2 * torch.randn(hd, generator=g, device=DEV)).to(dt)
    else:
        n, ctx = lengths(case)
        T, n_kv, hd = sum(n), case["n_kv"], case["hd"]
        s.update(_pages(case, n, ctx, g))
        s["err"] = torch.zeros(1, dtype=torch.int32, device=DEV)
        if case["kind"] == "append":
            row = _normal(g, T, 2 * n_kv, hd, dtype=DT[case["dtype"]])
            s.update(k=row[:, :n_kv], v=row[:, n_kv:])
            s["req"] = torch.repeat_interleave(torch.arange(len(n), dtype=torch.int32),
                                               torch.tensor(n)).to(DEV)
            s["pos"] = torch.cat([torch.arange(c, c + a, dtype=torch.int32)
                                  for a, c in zip(n, ctx)]).to(DEV)
        else:
            n_q = case["n_q"]
            s["q"] = _normal(g, T, n_q, hd, dtype=torch.bfloat16)
            at = [0]
            for a in n:
                at.append(at[-1] + a)
            s["cu"] = torch.tensor(at, dtype=torch.int32, device=DEV)
            s["kv_len"] = torch.tensor([a + c for a, c in zip(n, ctx)], dtype=torch.int32, device=DEV)
            s.update(n=n, total=[a + c for a, c in zip(n, ctx)], scale=hd ** -0.5, max_q=max(n),
                     out=torch.zeros(T, n_q, hd, dtype=torch.bfloat16, device=DEV),
                     lse=torch.zeros(n_q, T, dtype=torch.float32, device=DEV))
    if case.get("rot"):
        s["freq"] = _frequencies(case["rot"])
    if own:  # the descriptors and the workspace that a program keeps
        import paper_2607_22595_amd as xm
        pairing = xm.XMIX_ROPE_PAIRS if case.get("pairs") else xm.XMIX_ROPE_HALF
        s["xm"], s["rope"] = xm, xm.Rope(s["freq"], pairing) if case.get("rot") else None
        if case["kind"] != "norm_rope":
            s["cache"] = xm.KvCache(s["k_pages"], s["v_pages"], s["table"], s["k_scale"], s["v_scale"])
        if case["kind"] == "attend":
            s["ws"] = torch.empty(xm.paged_attention_workspace(T, case["n_q"], s["max_q"], s["cache"]),
                                  dtype=torch.uint8, device=DEV)
    return s


# -------------------------------------------------------------- the plain forms

def _rotate(x, pos, freq, pairs):
    """The first 2 * len(freq) values of each head turned by the position's angles
    (in 64 bits: a far position loses the angle in 32)."""
    angle = pos.double()[:, None] * freq
    c, s = angle.cos().float()[:, None], angle.sin().float()[:, None]
    rot = 2 * freq.numel()
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    a, b = a * c - b * s, b * c + a * s
    turned = torch.stack((a, b), -1).flatten(-2) if pairs else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., rot:]), -1)


def _plain_norm_rope(s):
    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + s["eps"]) * w.float()
        return _rotate(y, s["pos"], s["freq"], s["case"]["pairs"]).to(x.dtype)

    return one(s["q"], s["q_w"]), one(s["k"], s["k_w"])


def _plain_append(s):
    ps = s["case"]["page"]
    page = s["table"][s["req"].long(), (s["pos"] // ps).long()].long()
    slot = (s["pos"] % ps).long()
    k, v = s["k"].float(), s["v"].float()
    if s["case"]["rot"]:
        k = _rotate(k, s["pos"], s["freq"], s["case"]["pairs"])
    if s["k_scale"] is not None:
        k = (k / s["k_scale"][:, None]).clamp(-E4M3_MOST, E4M3_MOST)
        v = (v / s["v_scale"][:, None]).clamp(-E4M3_MOST, E4M3_MOST)
    dt = s["k_pages"].dtype
    bits = torch.uint8 if dt == torch.float8_e4m3fn else torch.int16
    s["k_pages"].view(bits)[page, :, slot] = k.to(dt).view(bits)
    s["v_pages"].view(bits)[page, :, slot] = v.to(dt).view(bits)
    return s["k_pages"], s["v_pages"]


def _plain_attend(s):
    # requests of one new token and of several each make a padded batch
    one = [r for r, a in enumerate(s["n"]) if a == 1]
    more = [r for r, a in enumerate(s["n"]) if a > 1]
    if one:
        _plain_batch(s, one)
    if more:
        _plain_batch(s, more)
    return s["out"], s["lse"]


def _plain_batch(s, reqs):
    case = s["case"]
    n_q, n_kv, hd, ps = case["n_q"], case["n_kv"], case["hd"], case["page"]
    n, B = max(s["n"][r] for r in reqs), len(reqs)
    keys = -(-max(s["total"][r] for r in reqs) // ps) * ps
    r = torch.tensor(reqs, device=DEV)
    first, end = s["cu"][r].long(), s["cu"][r + 1].long()
    token = first[:, None] + torch.arange(n, device=DEV)
    live = token < end[:, None]
    pos = s["kv_len"][r][:, None] - (end - first)[:, None] + torch.arange(n, device=DEV)
    page = s["table"][r][:, :keys // ps].clamp_min(0).long()

    def gather(pages, scale):
        x = pages.view(torch.uint8)[page].view(pages.dtype).float()
        x = x.permute(0, 2, 1, 3, 4).reshape(B, n_kv, keys, hd)
        return x if scale is None else x * scale[:, None, None]

    q = s["q"][torch.where(live, token, first[:, None])].float()
    q = q.view(B, n, n_kv, n_q // n_kv, hd).permute(0, 2, 3, 1, 4).reshape(B, n_kv, -1, hd)
    x = q @ gather(s["k_pages"], s["k_scale"]).transpose(-1, -2)
    x = (x * s["scale"]).view(B, n_kv, n_q // n_kv, n, keys)
    j = torch.arange(keys, device=DEV)
    seen = j <= pos[..., None]
    if case["window"]:
        seen &= j > pos[..., None] - case["window"]
    x = x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0.0, m)
    x = x.sub_(m).exp_()
    total = x.sum(-1, keepdim=True)
    o = x.view(B, n_kv, -1, keys) @ gather(s["v_pages"], s["v_scale"])
    o = o.view(B, n_kv, n_q // n_kv, n, hd) / torch.where(total == 0, 1.0, total)
    o = o.permute(0, 3, 1, 2, 4).reshape(B, n, n_q, hd)
    lse = (m + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(B, n, n_q)
    s["out"][token[live]] = o[live].to(torch.bfloat16)
    s["lse"][:, token[live]] = lse[live].t()


def _own(s):
    xm = s["xm"]
    kind = s["case"]["kind"]
    if kind == "norm_rope":
        xm.xmix_qk_norm_rope(s["q"], s["k"], s["pos"], s["q_w"], s["k_w"], s["eps"], s["rope"],
                             s["q_out"], s["k_out"])
        return s["q_out"], s["k_out"]
    if kind == "append":
        xm.xmix_kv_append(s["k"], s["v"], s["req"], s["pos"], s["rope"], s["cache"], s["err"])
        return s["k_pages"], s["v_pages"]
    xm.xmix_paged_attention(s["q"], s["cu"], s["kv_len"], s["cache"], s["scale"], s["case"]["window"],
                            s["max_q"], s["out"], s["lse"], s["err"], s["ws"])
    return s["out"], s["lse"]


def run(state):
    if own:
        return _own(state)
    kind = state["case"]["kind"]
    if kind == "norm_rope":
        return _plain_norm_rope(state)
    return _plain_append(state) if kind == "append" else _plain_attend(state)


# ---------------------------------------------------------------- in 64 bits

def _turn64(x, pos, freq, pairs):
    """The rotation as a product of complex numbers."""
    rot = 2 * freq.numel()
    z = x[..., :rot].unflatten(-1, (-1, 2) if pairs else (2, -1))
    z = torch.complex(z[..., 0], z[..., 1]) if pairs else torch.complex(z[..., 0, :], z[..., 1, :])
    angle = torch.outer(pos.double(), freq)
    parts = torch.view_as_real(z * torch.polar(torch.ones_like(angle), angle)[:, None])
    y = x.clone()
    y[..., :rot] = parts.flatten(-2) if pairs else parts.transpose(-1, -2).flatten(-2)
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "norm_rope":
        def one(x, w):
            y = x.double()
            if w is not None:
                length = (y.square().sum(-1) / case["hd"] + s["eps"]).sqrt()
                y = y / length[..., None] * w.double()
            return _turn64(y, s["pos"], s["freq"], case["pairs"])

        return one(s["q"], s["q_w"]), one(s["k"], s["k_w"])
    ps = case["page"]
    if case["kind"] == "append":
        k = s["k"].double()
        if case["rot"]:
            k = _turn64(k, s["pos"], s["freq"], case["pairs"])
        both = []
        for x, pages, scale in ((k, s["k_pages"], s["k_scale"]), (s["v"].double(), s["v_pages"], s["v_scale"])):
            y = pages.double()
            if scale is not None:
                x = (x / scale.double()[:, None]).clamp(-E4M3_MOST, E4M3_MOST)
            flat = y.permute(0, 2, 1, 3).reshape(-1, case["n_kv"], case["hd"])
            at = s["table"].long()[s["req"].long(), s["pos"].long() // ps] * ps + s["pos"].long() % ps
            flat[at] = x
            both.append(flat.view(y.shape[0], ps, case["n_kv"], case["hd"]).permute(0, 2, 1, 3).contiguous())
        return tuple(both)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device=DEV)
    G, at = case["n_q"] // case["n_kv"], 0
    for r, (n, total) in enumerate(zip(s["n"], s["total"])):
        page = s["table"][r, :-(-total // ps)].long()
        position = torch.arange(total - n, total, device=DEV)[:, None]
        key = torch.arange(total, device=DEV)
        hidden = (key > position) | ((key <= position - case["window"]) if case["window"] else False)
        for h in range(case["n_kv"]):
            k = s["k_pages"].view(torch.uint8)[page, h].view(s["k_pages"].dtype).double().flatten(0, 1)[:total]
            v = s["v_pages"].view(torch.uint8)[page, h].view(s["v_pages"].dtype).double().flatten(0, 1)[:total]
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"][h].double(), v * s["v_scale"][h].double()
            q = s["q"][at:at + n, h * G:(h + 1) * G].double().transpose(0, 1).reshape(G * n, -1)
            x = (s["scale"] * (q @ k.t())).view(G, n, total).masked_fill(hidden, -math.inf)
            z = torch.logsumexp(x, -1)
            o = (x - z[..., None]).exp().view(G * n, total) @ v
            out[at:at + n, h * G:(h + 1) * G] = o.view(G, n, -1).transpose(0, 1)
            lse[h * G:(h + 1) * G, at:at + n] = z
        at += n
    return out, lse
