"""The serving operators on a caller's own tensors, as cases to be timed: rotary positions, rotary positions with the append to a
paged key-value cache, attention of new tokens over such a cache, and verification of drafted tokens from given probabilities and
random numbers.  Together they are a target model's step around its matrix products.

Head layouts, page size, draft lengths and vocabularies are those of this repository's workloads (`ssd_inputs`): the tiny fp32 pair (4 / 4
heads of 64), the Llama-3.2-1B-shaped draft (32 / 8 heads of 64), the Llama-3.1-70B-shaped target (64 / 8 heads of 128); drawn cases
take other layouts too.  With `own` false a pass is the operators' plain form in elementary torch operations, with `own` true the
library's calls."""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
PLAIN, LINEAR, BANDS, RAMP = "plain", "linear", "bands", "ramp"


def listed():
    return [
        # ---- rotary positions alone
        # queries of a small batch of the tiny pair: interleaved pairs in half of the head, latency
        dict(name="rope_r15_tiny_f32", kind="rope", dtype="f32", rows=15, H=4, D=64, rot=32, layout="interleaved", scaling=PLAIN, pos=100),
        # queries and keys of a long prompt, far positions, stretched frequencies
        dict(name="rope_r2039_h72_d128", kind="rope", dtype="bf16", rows=2039, H=72, D=128, rot=128, layout="half", scaling=RAMP, pos=120000),
        # ---- rotary positions and the append to the cache
        # one new token of one sequence: the smallest decode step
        dict(name="append_b1_t1_1b", kind="append", dtype="bf16", cache="bf16", B=1, T=1, Hq=32, Hkv=8, D=64, rot=64, layout="half",
             scaling=BANDS, pos=1024, page=32),
        # a batch's verification blocks of unequal length, fp32 projections into a bf16 cache
        dict(name="append_b16_t6_70b", kind="append", dtype="f32", cache="bf16", B=16, T=6, Hq=64, Hkv=8, D=128, rot=128, layout="half",
             scaling=BANDS, pos=2500, page=32, ragged=True),
        # a prompt's prefill in one pass
        dict(name="append_b1_t4093_70b", kind="append", dtype="bf16", cache="bf16", B=1, T=4093, Hq=64, Hkv=8, D=128, rot=128, layout="half",
             scaling=PLAIN, pos=0, page=32),
        # ---- attention over the paged cache
        # the tiny fp32 pair's verification block: everything is launches and latency
        dict(name="attn_b1_t5_p128_tiny", kind="attn", dtype="f32", cache="f32", B=1, T=5, Hq=4, Hkv=4, D=64, P=133, page=32),
        # the target verifies K = 5 drafted tokens of one sequence
        dict(name="attn_b1_t6_p4096_70b", kind="attn", dtype="bf16", cache="bf16", B=1, T=6, Hq=64, Hkv=8, D=128, P=4102, page=32),
        # a draft's branches: 24 rows that share a long trunk, each with private keys behind it; fp32 queries as the library's passes have
        dict(name="attn_b1_r24_p8192_tails", kind="attn", dtype="f32", cache="bf16", B=1, T=24, Hq=32, Hkv=8, D=64, P=8198, page=32, tail=5),
        # a serving batch of 16 with a prefix length per sequence, one slot empty, small pages
        dict(name="attn_b16_t6_p2048_ragged", kind="attn", dtype="bf16", cache="bf16", B=16, T=6, Hq=32, Hkv=8, D=64, P=2054, page=16, ragged=True),
        # one new token each for a large batch of long sequences
        dict(name="attn_b64_t1_p8192_70b", kind="attn", dtype="bf16", cache="bf16", B=64, T=1, Hq=64, Hkv=8, D=128, P=8193, page=32),
        # ---- verification from given probabilities and random numbers
        dict(name="verify_b1_k5", kind="verify", B=1, K=5, V=128256),
        dict(name="verify_b64_k7_ragged", kind="verify", B=64, K=7, V=128256, ragged=True),
    ]


LAYOUTS = [(32, 8, 64), (64, 8, 128), (4, 4, 64), (8, 1, 128), (12, 2, 64), (28, 4, 128), (16, 16, 128), (40, 8, 128)]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_rotation(rng, D):
    rot = rng.choice([D, D, D // 2, D // 4, 3 * D // 4])
    return dict(rot=rot, layout=rng.choice(["half", "half", "interleaved"]), scaling=rng.choice([PLAIN, LINEAR, BANDS, RAMP]))


def draw(rng):
    most = {}
    for c in listed():
        most[c["kind"]] = max(most.get(c["kind"], 0.0), work(c)["bytes"])
    while True:
        kind = rng.choice(["rope", "append", "append", "attn", "attn", "attn", "verify", "verify"])
        hq, hkv, d = rng.choice(LAYOUTS)
        if kind == "rope":
            c = dict(kind=kind, dtype=rng.choice(["f32", "bf16"]), rows=_log_int(rng, 1, 2000), H=rng.choice([hq, hq + hkv]), D=d,
                     pos=_log_int(rng, 1, 200000), **_draw_rotation(rng, d))
        elif kind == "append":
            t = rng.choice([1, rng.randint(1, 16), _log_int(rng, 16, 4000)])
            c = dict(kind=kind, B=_log_int(rng, 1, 64 if t <= 16 else 4), T=t, Hq=hq, Hkv=hkv, D=d, pos=_log_int(rng, 1, 50000) if t <= 16 else 0,
                     page=rng.choice([8, 16, 32, 64]), ragged=rng.random() < 0.5, **_draw_rotation(rng, d))
            c["dtype"], c["cache"] = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
        elif kind == "attn":
            c = dict(kind=kind, B=_log_int(rng, 1, 64), T=rng.choice([1, 1, rng.randint(2, 8), rng.randint(9, 40)]), Hq=hq, Hkv=hkv, D=d,
                     P=_log_int(rng, 1, 32768), page=rng.choice([8, 16, 32, 64]), ragged=rng.random() < 0.5)
            c["dtype"], c["cache"] = rng.choice([("bf16", "bf16"), ("bf16", "bf16"), ("f32", "bf16"), ("f32", "f32")])
            if rng.random() < 0.3:
                c["tail"] = rng.randint(1, 8)
            # (the plain form holds a batch's cache and scores in 32 bits)
            if c["B"] * c["P"] * (hkv * d + hq * c["T"]) > 600e6:
                continue
        else:
            c = dict(kind=kind, B=_log_int(rng, 1, 64), K=rng.randint(1, 15), V=rng.choice([128256, 32003, 50257, _log_int(rng, 100, 100000)]),
                     ragged=rng.random() < 0.5, one_hot=rng.random() < 0.2)
            if c["B"] * (c["K"] + 1) * c["V"] > 64 * 8 * 128256:
                continue
        if work(c)["bytes"] <= most[kind]:
            return c


# ------------------------------------------------------------------------------------------------ what a pass needs

def _lens(c):
    """Positions of the cache every sequence has when its new tokens are in: the same, or from none to P."""
    if not c.get("ragged"):
        return [c["P"]] * c["B"]
    return [c["P"]] + [c["P"] * ((7 * b) % c["B"]) // c["B"] if b != c["B"] // 2 else 0 for b in range(1, c["B"])]


def _visible(c):
    """Positions that each row sees, [B][T]: a block's tokens see one another causally, branches the trunk up to their fork."""
    n = torch.tensor(_lens(c)).unsqueeze(1)
    t = torch.arange(c["T"]).unsqueeze(0)
    back = t % 6 if c.get("tail") else c["T"] - 1 - t
    return (n - back).clamp(min=0)


def _new_tokens(c):
    """New tokens of each sequence: T, or from one to T."""
    return [c["T"] if not c.get("ragged") else 1 + (c["T"] - 1) * ((5 * b) % c["B"]) // max(1, c["B"] - 1) for b in range(c["B"])]


def _drafted(c):
    return [c["K"] if not c.get("ragged") else (3 * b + c["K"]) % (c["K"] + 1) for b in range(c["B"])]


def _size(dtype):
    return 4 if dtype == "f32" else 2


def work(case):
    c = case
    if c["kind"] == "rope":
        n = c["rows"] * c["H"]
        return {"bytes": 2.0 * n * c["D"] * _size(c["dtype"]) + 4.0 * c["rows"], "flops": 3.0 * n * c["rot"]}
    if c["kind"] == "append":
        rows, kept = c["B"] * c["T"], sum(_new_tokens(c))
        es, ec = _size(c["dtype"]), _size(c["cache"])
        by = rows * 2 * c["Hq"] * c["D"] * es + kept * 2 * c["Hkv"] * c["D"] * (es + ec) + rows * 8
        return {"bytes": float(by), "flops": 3.0 * (rows * c["Hq"] + kept * c["Hkv"]) * c["rot"]}
    if c["kind"] == "attn":
        vis = _visible(c)
        seen, tail = int(vis.max(dim=1).values.sum()), c.get("tail", 0)
        rows = c["B"] * c["T"]
        by = (seen + rows * tail) * 2 * c["Hkv"] * c["D"] * _size(c["cache"]) + 2 * rows * c["Hq"] * c["D"] * _size(c["dtype"]) + 4 * rows
        return {"bytes": float(by), "flops": 4.0 * c["Hq"] * c["D"] * (int(vis.sum()) + rows * tail)}
    # a token drafted from a distribution this near the target's is accepted seven times in ten: the target's row that decides is read
    # once, the draft's where a token was rejected
    rejected = [0.0 if c.get("one_hot") else 1.0 - 0.7 ** n for n in _drafted(c)]
    rows = sum(1.0 + r for r in rejected)
    return {"bytes": 4.0 * c["V"] * rows + 16.0 * c["B"] * c["K"], "flops": 3.0 * c["V"] * rows}


# ------------------------------------------------------------------------------------------------ states

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed) & 0x7FFFFFFF)


def _ints(v):
    return torch.as_tensor(v, dtype=torch.int32).cuda()


def _rotation(c):
    """theta, factor, low, high, original context, magnitude of a case's scaling"""
    return {PLAIN: (10000.0, 1.0, 0.0, 0.0, 0.0, 1.0), LINEAR: (10000.0, 4.0, 0.0, 0.0, 0.0, 1.0),
            BANDS: (500000.0, 32.0, 1.0, 4.0, 8192.0, 1.0), RAMP: (500000.0, 16.0, 1.0, 32.0, 8192.0, 1.277)}[c["scaling"]]


def _table(g, needed, blocks, spare):
    """A pool's pages dealt to the blocks of each sequence in a shuffled order: table [B][blocks] (-1: no page), pages in the pool."""
    used = torch.zeros((len(needed), blocks), dtype=torch.bool)
    for b, (lo, hi) in enumerate(needed):
        used[b, lo:hi] = True
    n = int(used.sum())
    table = torch.full((len(needed), blocks), -1, dtype=torch.int32, device="cuda")
    table[used.cuda()] = torch.randperm(n + spare, generator=g, device="cuda")[:n].to(torch.int32)
    return table.contiguous(), n + spare


def prepare(case, seed):
    c, g = case, _generator(seed)
    s = {"case": c}

    def normal(shape, dtype):
        return torch.randn(shape, generator=g, device="cuda").to(DTYPES[dtype])

    if c["kind"] == "rope":
        s["x"] = normal((c["rows"], c["H"], c["D"]), c["dtype"])
        s["positions"] = (c["pos"] + torch.arange(c["rows"], device="cuda")).to(torch.int32)
        s["out"] = torch.empty_like(s["x"])
        return s
    if c["kind"] == "append":
        nb, T, hq, hkv, d, page = (c[k] for k in ("B", "T", "Hq", "Hkv", "D", "page"))
        # the projections as one matrix product leaves them
        qkv = normal((nb, T, (hq + 2 * hkv) * d), c["dtype"])
        q, k, v = qkv.split([hq * d, hkv * d, hkv * d], dim=2)
        s["q"], s["k"], s["v"] = q.unflatten(2, (hq, d)), k.unflatten(2, (hkv, d)), v.unflatten(2, (hkv, d))
        start = torch.tensor([c["pos"] + (37 * b) % 101 for b in range(nb)])
        positions = start.unsqueeze(1) + torch.arange(T).unsqueeze(0)
        kept = torch.arange(T).unsqueeze(0) < torch.tensor(_new_tokens(c)).unsqueeze(1)
        s["positions"] = _ints(positions)
        s["slots"] = _ints(torch.where(kept, positions, -1))       # rows behind a sequence's own tokens pad the batch
        # (the call does not touch the pages of earlier positions: the case keeps none)
        first, last = start // page, (start + T - 1) // page + 1
        s["table"], n = _table(g, list(zip(first.tolist(), last.tolist())), int(last.max()), 2)
        # the last page is nobody's: the plain form stores rows there that pad
        s["pool_k"] = normal((n + 1, page, hkv, d), c["cache"])
        s["pool_v"] = normal((n + 1, page, hkv, d), c["cache"])
        s["q_out"] = torch.empty((nb, T, hq, d), dtype=DTYPES[c["dtype"]], device="cuda")
        return s
    if c["kind"] == "attn":
        nb, T, hq, hkv, d, page = (c[k] for k in ("B", "T", "Hq", "Hkv", "D", "page"))
        blocks = max(1, -(-c["P"] // page))
        s["table"], n = _table(g, [(0, -(-x // page)) for x in _lens(c)], blocks, 2)
        s["pool_k"] = normal((n, page, hkv, d), c["cache"])
        s["pool_v"] = normal((n, page, hkv, d), c["cache"])
        s["q"] = normal((nb, T, hq, d), c["dtype"])
        s["visible"] = _ints(_visible(c))
        s["out"] = torch.empty((nb, T, hq, d), dtype=DTYPES[c["dtype"]], device="cuda")
        if c.get("tail"):
            # room for two more tokens than the rows have yet
            s["tail_k"] = normal((nb, T, c["tail"] + 2, hkv, d), c["cache"])
            s["tail_v"] = normal((nb, T, c["tail"] + 2, hkv, d), c["cache"])
        return s
    nb, K, V = c["B"], c["K"], c["V"]
    # a draft that is close to the target, and tokens drawn from it
    base = torch.randn((nb, K + 1, V), generator=g, device="cuda") * 2.5
    s["target"] = torch.softmax(base + 0.5 * torch.randn((nb, K + 1, V), generator=g, device="cuda"), dim=2)
    draft = torch.softmax(base[:, :K] + 0.5 * torch.randn((nb, K, V), generator=g, device="cuda"), dim=2)
    s["spec"] = torch.multinomial(draft.reshape(nb * K, V), 1, generator=g).reshape(nb, K).to(torch.int32)
    s["draft"] = None if c.get("one_hot") else draft        # a lookup's tokens come without probabilities
    s["drafted"] = _ints(_drafted(c))
    s["u_accept"] = torch.rand((nb, K), generator=g, device="cuda")
    s["u_bonus"] = torch.rand((nb,), generator=g, device="cuda")
    s["accept_len"] = torch.empty(nb, dtype=torch.int32, device="cuda")
    s["bonus"] = torch.empty(nb, dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _frequencies(c):
    """Angle per position of each pair of a head, fp64 on the GPU."""
    theta, factor, low, high, original, _ = _rotation(c)
    i = torch.arange(c["rot"] // 2, dtype=torch.float64, device="cuda")
    f = torch.exp(i * (-2.0 / c["rot"] * math.log(theta)))
    if c["scaling"] == LINEAR:
        return f / factor
    if c["scaling"] == BANDS:       # by the turns a pair makes over the original context
        keep = ((original * f / (2.0 * math.pi) - low) / (high - low)).clamp(0.0, 1.0)
        return f * (keep + (1.0 - keep) / factor)
    if c["scaling"] == RAMP:        # by the index of the pair, between those of `high` and `low` turns
        def index(turns):
            return c["rot"] * math.log(original / (2.0 * math.pi * turns)) / (2.0 * math.log(theta))
        i0, i1 = max(math.floor(index(high)), 0), min(math.ceil(index(low)), c["rot"] - 1)
        slow = ((i - i0) / max(i1 - i0, 1e-3)).clamp(0.0, 1.0)
        return f * (1.0 - slow + slow / factor)
    return f


def _rotate(c, x, positions):
    """x [..][H][D] in 32 bits, positions [..]; angles in 64"""
    angle = (positions.double().unsqueeze(-1) * _frequencies(c)).unsqueeze(-2)
    magnitude = _rotation(c)[5]
    cos, sin = (torch.cos(angle) * magnitude).float(), (torch.sin(angle) * magnitude).float()
    x = x.float()
    turned, rest = x[..., :c["rot"]], x[..., c["rot"]:]
    if c["layout"] == "half":
        a, b = turned.chunk(2, dim=-1)
        return torch.cat([a * cos - b * sin, b * cos + a * sin, rest], dim=-1)
    a, b = turned[..., 0::2], turned[..., 1::2]
    return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2), rest], dim=-1)


def _plain_append(s, c):
    page = c["page"]
    s["q_out"].copy_(_rotate(c, s["q"], s["positions"]))
    slots = s["slots"].long()
    at = torch.gather(s["table"].long(), 1, slots.clamp(min=0) // page) * page + slots.clamp(min=0) % page
    nobody = (s["pool_k"].shape[0] - 1) * page
    at = torch.where(slots >= 0, at, nobody).flatten()
    s["pool_k"].flatten(0, 1).index_put_((at,), _rotate(c, s["k"], s["positions"]).to(s["pool_k"].dtype).flatten(0, 1))
    s["pool_v"].flatten(0, 1).index_put_((at,), s["v"].to(s["pool_v"].dtype).flatten(0, 1))
    return {"q": s["q_out"], "k": s["pool_k"][:-1], "v": s["pool_v"][:-1]}


def _plain_attention(s, c):
    nb, T, hq, hkv, d = (c[k] for k in ("B", "T", "Hq", "Hkv", "D"))
    G = hq // hkv
    table = s["table"].long().clamp(min=0)
    heads = [p[table].flatten(1, 2).permute(0, 2, 1, 3).float() for p in (s["pool_k"], s["pool_v"])]       # [B][Hkv][positions][D]
    q = s["q"].float().reshape(nb, T, hkv, G, d).permute(0, 2, 1, 3, 4).reshape(nb, hkv, T * G, d)
    scores = torch.matmul(q, heads[0].transpose(2, 3).contiguous()) / math.sqrt(d)
    sees = torch.arange(scores.shape[3], device="cuda") < s["visible"].repeat_interleave(G, dim=1)[:, None, :, None]
    scores = torch.where(sees, scores, -math.inf)
    if c.get("tail"):
        n = c["tail"]
        tk, tv = (t[:, :, :n].float().permute(0, 3, 1, 2, 4) for t in (s["tail_k"], s["tail_v"]))             # [B][Hkv][T][n][D]
        own_scores = torch.matmul(q.unflatten(2, (T, G)), tk.transpose(3, 4).contiguous()).flatten(2, 3) / math.sqrt(d)
        scores = torch.cat([scores, own_scores], dim=3)
    top = scores.amax(dim=3, keepdim=True)
    p = torch.exp(scores - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(dim=3, keepdim=True)
    o = torch.matmul(p[..., :heads[1].shape[2]], heads[1])
    if c.get("tail"):
        o = o + torch.matmul(p[..., heads[1].shape[2]:].unflatten(2, (T, G)), tv).flatten(2, 3)
    o = torch.where(total > 0, o / total, 0.0)
    s["out"].copy_(o.reshape(nb, hkv, T, G, d).permute(0, 2, 1, 3, 4).reshape(nb, T, hq, d))
    return s["out"]


def _plain_verify(s, c):
    nb, K = c["B"], c["K"]
    spec = s["spec"].long().unsqueeze(2)
    p = torch.gather(s["target"][:, :K], 2, spec).squeeze(2).double()
    q = torch.ones_like(p) if s["draft"] is None else torch.gather(s["draft"], 2, spec).squeeze(2).double()
    drafted = torch.arange(K, device="cuda") < s["drafted"].unsqueeze(1)
    ok = (s["u_accept"].double() * q < p) & drafted
    s["accept_len"].copy_(ok.int().cumprod(dim=1).sum(dim=1))
    k, b = s["accept_len"].long(), torch.arange(nb, device="cuda")
    row = s["target"][b, k].double()
    at = k.clamp(max=K - 1)
    if s["draft"] is None:
        less = torch.zeros_like(row).scatter_(1, spec[b, at], 1.0)
    else:
        less = s["draft"][b, at].double()
    left = torch.where((k < s["drafted"]).unsqueeze(1), (row - less).clamp(min=0.0), row)
    left = torch.where(left.sum(dim=1, keepdim=True) > 0, left, row)
    upto = left.cumsum(dim=1)
    s["bonus"].copy_((upto <= s["u_bonus"].double().unsqueeze(1) * upto[:, -1:]).sum(dim=1))
    return {"accept_len": s["accept_len"], "bonus": s["bonus"]}


# ------------------------------------------------------------------------------------------------ passes

def _own_rope(s, c):
    from paper_2603_03251_amd import binding as B
    if "rope" not in s:
        theta, factor, low, high, original, magnitude = _rotation(c)
        s["rope"] = B.rope_config(theta, c["rot"], layout=c["layout"], scaling=c["scaling"], factor=factor, low=low, high=high,
                                  original=original, magnitude=magnitude)
    return B


def run(state):
    s, c = state, state["case"]
    if c["kind"] == "rope":
        if own:
            B = _own_rope(s, c)
            B.ssd_rope(s["rope"], s["x"], s["positions"], s["out"])
            return s["out"]
        s["out"].copy_(_rotate(c, s["x"], s["positions"]))
        return s["out"]
    if c["kind"] == "append":
        if own:
            B = _own_rope(s, c)
            if "kv" not in s:
                s["kv"] = B.paged_kv(s["pool_k"][:-1], s["pool_v"][:-1], s["table"])
            B.ssd_rope_append(s["rope"], s["q"], s["k"], s["v"], s["positions"], s["kv"], s["q_out"], slots=s["slots"])
            return {"q": s["q_out"], "k": s["pool_k"][:-1], "v": s["pool_v"][:-1]}
        return _plain_append(s, c)
    if c["kind"] == "attn":
        if own:
            from paper_2603_03251_amd import binding as B
            tail = c.get("tail", 0)
            if "kv" not in s:
                s["kv"] = B.paged_kv(s["pool_k"], s["pool_v"], s["table"])
                n = B.ssd_paged_attention_workspace_bytes(s["kv"], c["B"], c["T"], c["Hq"], c["P"])
                s["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
                s["tails"] = B.tail_kv(s["tail_k"], s["tail_v"], tail) if tail else None
            B.ssd_paged_attention(s["kv"], s["q"], s["visible"], c["P"], s["out"], s["workspace"], tail=s["tails"])
            return s["out"]
        return _plain_attention(s, c)
    if own:
        from paper_2603_03251_amd import binding as B
        if "workspace" not in s:
            s["workspace"] = torch.empty(B.ssd_verify_probs_workspace_bytes(c["B"], c["V"]), dtype=torch.uint8, device="cuda")
        B.ssd_verify_probs(s["target"], s["draft"], s["spec"], s["u_accept"], s["u_bonus"], s["accept_len"], s["bonus"], s["workspace"],
                           drafted=s["drafted"])
        return {"accept_len": s["accept_len"], "bonus": s["bonus"]}
    return _plain_verify(s, c)


# ------------------------------------------------------------------------------------------------ from the definitions, in 64 bits

def _exact_rotation(c, x, positions):
    """Pair (a, b) as the complex number a + ib, times exp(i position f)."""
    theta, factor, low, high, original, magnitude = _rotation(c)
    rot = c["rot"]
    freq = []
    for i in range(rot // 2):
        f = theta ** (-2.0 * i / rot)
        if c["scaling"] == LINEAR:
            f /= factor
        elif c["scaling"] == BANDS:
            wave = 2.0 * math.pi / f
            if wave > original / low:
                f /= factor
            elif wave >= original / high:
                mix = (original / wave - low) / (high - low)
                f = (1.0 - mix) * f / factor + mix * f
        elif c["scaling"] == RAMP:
            lo = max(math.floor(rot / 2.0 * math.log(original / (high * 2.0 * math.pi)) / math.log(theta)), 0)
            hi = min(math.ceil(rot / 2.0 * math.log(original / (low * 2.0 * math.pi)) / math.log(theta)), rot - 1)
            share = 1.0 - min(max((i - lo) / (hi - lo if hi > lo else 1e-3), 0.0), 1.0)
            f = f / factor * (1.0 - share) + f * share
        freq.append(f)
    angle = positions.to(torch.float64)[..., None, None] * torch.tensor(freq, dtype=torch.float64, device="cuda")
    turn = torch.polar(torch.full_like(angle, magnitude), angle)
    y = x.to(torch.float64).clone()
    if c["layout"] == "half":
        z = torch.complex(y[..., :rot // 2].clone(), y[..., rot // 2:rot].clone()) * turn
        y[..., :rot // 2], y[..., rot // 2:rot] = z.real, z.imag
    else:
        z = torch.complex(y[..., 0:rot:2].clone(), y[..., 1:rot:2].clone()) * turn
        y[..., 0:rot:2], y[..., 1:rot:2] = z.real, z.imag
    return y


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "rope":
        return _exact_rotation(c, s["x"], s["positions"])
    if c["kind"] == "append":
        pools = {"k": s["pool_k"][:-1].to(torch.float64), "v": s["pool_v"][:-1].to(torch.float64)}
        k = _exact_rotation(c, s["k"], s["positions"])
        for b, n in enumerate(_new_tokens(c)):
            t = s["positions"][b, :n].long()
            page = s["table"][b].long()[t // c["page"]]
            pools["k"][page, t % c["page"]] = k[b, :n]
            pools["v"][page, t % c["page"]] = s["v"][b, :n].to(torch.float64)
        return {"q": _exact_rotation(c, s["q"], s["positions"]), **pools}
    if c["kind"] == "attn":
        T, hq, hkv, d = c["T"], c["Hq"], c["Hkv"], c["D"]
        out = torch.zeros((c["B"], T, hq, d), dtype=torch.float64, device="cuda")
        tail, vis = c.get("tail", 0), _visible(c)
        for b in range(c["B"]):
            n = int(vis[b].max())
            pages = s["table"][b, :-(-n // c["page"])].long()
            k, v = (s[p][pages].reshape(-1, hkv, d)[:n].to(torch.float64) for p in ("pool_k", "pool_v"))
            late = torch.arange(n, device="cuda").unsqueeze(0) >= vis[b].cuda().unsqueeze(1)
            late = torch.cat([late, torch.zeros((T, tail), dtype=torch.bool, device="cuda")], dim=1)
            if not n + tail:
                continue
            for h in range(hq):
                kv = h * hkv // hq
                q = s["q"][b, :, h].to(torch.float64) / math.sqrt(d)
                w = q @ k[:, kv].T
                if tail:
                    w = torch.cat([w, (q.unsqueeze(1) * s["tail_k"][b, :, :tail, kv].to(torch.float64)).sum(dim=2)], dim=1)
                w = torch.nan_to_num(torch.softmax(w.masked_fill(late, -math.inf), dim=1))
                out[b, :, h] = w[:, :n] @ v[:, kv]
                if tail:
                    out[b, :, h] += (w[:, n:].unsqueeze(2) * s["tail_v"][b, :, :tail, kv].to(torch.float64)).sum(dim=1)
        return out
    lens, bonus = [], []
    for b, drafted in enumerate(_drafted(c)):
        k = 0
        while k < drafted:
            t = int(s["spec"][b, k])
            q = 1.0 if s["draft"] is None else float(s["draft"][b, k, t])
            if not float(s["u_accept"][b, k]) * q < float(s["target"][b, k, t]):
                break
            k += 1
        mass = s["target"][b, k].to(torch.float64).clone()
        if k < drafted:
            if s["draft"] is None:
                mass[int(s["spec"][b, k])] = 0.0
            else:
                mass = torch.relu(mass - s["draft"][b, k].to(torch.float64))
        below = torch.cumsum(mass, dim=0)
        edge = float(s["u_bonus"][b]) * float(below[-1])
        lens.append(k)
        bonus.append(int(torch.searchsorted(below, torch.tensor([edge], dtype=torch.float64, device="cuda"), right=True)))
    return {"accept_len": torch.tensor(lens, dtype=torch.int32, device="cuda"), "bonus": torch.tensor(bonus, dtype=torch.int32, device="cuda")}
