"""Attention of grouped heads over a paged cache of keys and values, as cases that can be timed and compared.

A case is a dict of plain values.  Its "op" says which operator one pass runs:

  norm_rotary  tpla_norm_rotary_heads: every head of the queries and keys is normed (mean square, a weight per column) and
               turned to its token's position, in one pass.  Both are views into one projection [T, (H + 2 H_kv) d].
  append       tpla_append_heads: the same for the queries and keys of new tokens, the keys and the values written to their
               slots of the paged cache on the way.
  decode       tpla_decode_heads: one new token per sequence attends to all tokens of its sequence in the cache, H / H_kv
               query heads to each head of keys and values.
  prefill      tpla_prefill_heads: the new tokens of every sequence, packed, attend to what the cache holds of their sequence
               up to themselves: whole prompts, or parts of prompts behind cached tokens.

Where `own` is false the plain form of the operator runs: elementary torch operations in 32 bits (angles in 64).
"""
import math

import torch

own = False

DEFAULTS = dict(H=32, H_kv=8, d=128, dtype="bf16", page=64)
MOST_SCORES = 32 * 16384 * 16384                 # scores of the largest listed prefill case, masked ones included
MOST_CACHED = 2.0 * 8 * 128 * 48 * 7600          # cached values of the largest listed decode case
EPS = 1e-6


def listed():
    return [
        # one user's next token
        dict(name="norm_rotary_one", op="norm_rotary", T=1, layout="half", far=120000),
        # a batch of prompts before the attention of a layer: all bandwidth, an odd number of tokens
        dict(name="norm_rotary_prompts", op="norm_rotary", T=16411, layout="half", far=32768),
        # one new token for each of 61 running sequences, into a cache of 64-token pages
        dict(name="append_decode", op="append", T=61, layout="half", far=20000),
        # prompts of a model with many narrow heads and interleaved pairs, half of each head turned, pages of 16 tokens, some
        # tokens without a slot (their pages ran out)
        dict(name="append_prompts", op="append", T=9001, H=48, H_kv=12, d=64, rot=32, layout="interleaved", page=16, far=9001, skip=True),
        # the checks of a float model: a few tokens, three query heads to a head of keys, a width of no power of two
        dict(name="decode_f32_tiny", op="decode", B=3, min_len=1, max_len=70, H=6, H_kv=2, d=96, dtype="f32", page=16),
        # one user's conversation: all latency, work split over the length
        dict(name="decode_one_user", op="decode", B=1, min_len=9001, max_len=9001),
        # a serving batch of uneven lengths: all bandwidth
        dict(name="decode_ragged", op="decode", B=48, min_len=500, max_len=32000),
        # all query heads share one head of keys and values, small pages
        dict(name="decode_shared_head", op="decode", B=40, min_len=300, max_len=8000, H=16, H_kv=1, d=64, page=16),
        # float prompts
        dict(name="prefill_f32", op="prefill", B=3, min_new=30, max_new=300, min_len=0, max_len=150, H=6, H_kv=2, d=96, dtype="f32", page=16),
        # prompts of many lengths admitted at once, packed, nothing in the cache before
        dict(name="prefill_prompts", op="prefill", B=13, min_new=5, max_new=3001, min_len=0, max_len=0),
        # the next parts of two long prompts behind their cached tokens: few rows, many keys
        dict(name="prefill_part", op="prefill", B=2, min_new=200, max_new=512, min_len=8000, max_len=20011),
        # one long prompt: all matrix products
        dict(name="prefill_long", op="prefill", B=1, min_new=16384, max_new=16384, min_len=0, max_len=0),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm_rotary", "append", "decode", "decode", "decode", "prefill", "prefill", "prefill"])
    d, rows = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 4, 5, 8, 16])
    H_kv = rng.choice([1, 2, 4, 8, 8])
    c = dict(op=op, H=rows * H_kv, H_kv=H_kv, d=d, page=rng.choice([16, 32, 64, 64, 128]))
    if op in ("norm_rotary", "append"):
        c.update(T=_log_uniform(rng, 1, 10000), rot=rng.choice([d, d, d // 2]), layout=rng.choice(["interleaved", "half", "half"]),
                 far=_log_uniform(rng, 100, 1000000), dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]))
        c["T"] = max(1, min(c["T"], int(16411 * 40 * 128 / ((c["H"] + 2 * H_kv) * d * (2 if c["dtype"] == "f32" else 1)))))
        if op == "append":
            c["skip"] = rng.random() < 0.3
        return c
    if rng.random() < 0.12:                      # float models: small
        c.update(H=rng.choice([1, 2, 3]) * 2, H_kv=2, d=rng.choice([32, 64, 96]), dtype="f32", B=rng.randint(1, 6), max_len=_log_uniform(rng, 1, 600))
        c["min_len"] = max(1, c["max_len"] // 4)
        if op == "prefill":
            c["max_new"] = _log_uniform(rng, 1, 300)
            c["min_new"] = max(1, c["max_new"] // 5)
        return c
    hi = _log_uniform(rng, 1, 32768)
    if op == "decode":
        c.update(B=_log_uniform(rng, 1, 128), min_len=max(1, hi // rng.randint(1, 16)), max_len=hi)
        while c["B"] > 1 and 2.0 * H_kv * d * c["B"] * hi > MOST_CACHED:
            c["B"] = c["B"] * 2 // 3
        return c
    c.update(B=_log_uniform(rng, 1, 24), max_new=_log_uniform(rng, 2, 8192), max_len=rng.choice([0, 0, 1]) * hi)
    while c["H"] * c["B"] * c["max_new"] * (c["max_new"] + c["max_len"]) > MOST_SCORES:
        if c["B"] > 1:
            c["B"] = c["B"] * 2 // 3
        else:
            c["max_new"] = c["max_new"] * 2 // 3
    c["min_new"], c["min_len"] = max(1, c["max_new"] // rng.randint(1, 16)), c["max_len"] // rng.randint(1, 8)
    return c


# ------------------------------------------------------------------ inputs
class _Case:
    def __init__(self, case):
        for k, v in {**DEFAULTS, **case}.items():
            setattr(self, k, v)
        self.st = torch.float32 if self.dtype == "f32" else torch.bfloat16
        self.esz = 4 if self.dtype == "f32" else 2
        self.scale = 1.0 / math.sqrt(self.d)
        self.group = self.H // self.H_kv
        if self.op in ("norm_rotary", "append"):
            self.rot = getattr(self, "rot", self.d)
            return
        self.lens = _spread(self.min_len, self.max_len, self.B)              # tokens in the cache before the new ones of a prefill
        self.news = _spread(self.min_new, self.max_new, self.B)[::-1] if self.op == "prefill" else [0] * self.B
        self.keys = [a + b for a, b in zip(self.lens, self.news)]
        self.pages = [-(-n // self.page) for n in self.keys]
        self.max_pages = max(self.pages)
        self.T = sum(self.news)


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly over the logarithm (0 counts as below 1), in an order that mixes them."""
    v = [min(hi, max(lo, int((lo + 0.5) * ((hi + 0.5) / (lo + 0.5)) ** (i / max(1, n - 1))))) for i in range(n - 1)] + [hi]
    step = next(s for s in range(n // 2 + 1, 2 * n + 2) if math.gcd(s, n) == 1)
    return [v[(i * step + n - 1) % n] for i in range(n)]


def prepare(case, seed):
    c = _Case(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    normal = lambda *n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    empty = lambda *n: torch.empty(n, dtype=c.st, device="cuda")  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731

    def pool(n_pages):
        p = empty(n_pages, c.H_kv, c.page, c.d)
        for i in range(0, n_pages, 1024):
            p[i:i + 1024] = normal(*p[i:i + 1024].shape).to(c.st)
        return p

    if c.op in ("norm_rotary", "append"):
        qkv = (normal(c.T, c.H + 2 * c.H_kv, c.d) * 1.5).to(c.st)            # the projection of the block's input
        s = dict(q=qkv[:, :c.H], k=qkv[:, c.H:c.H + c.H_kv], v=qkv[:, c.H + c.H_kv:], q_out=empty(c.T, c.H, c.d),
                 w_q=(1 + 0.1 * normal(c.d)).to(c.st), w_k=(1 + 0.1 * normal(c.d)).to(c.st),
                 freq=500000.0 ** (-2.0 * torch.arange(c.rot // 2, dtype=torch.float64, device="cuda") / c.rot),
                 positions=torch.randint(0, c.far, (c.T,), generator=gen, device="cuda").to(torch.int32))
        if c.op == "norm_rotary":
            s["k_out"] = empty(c.T, c.H_kv, c.d)
        else:
            n_pages = c.T // c.page + 4
            s["k_pool"], s["v_pool"] = pool(n_pages), pool(n_pages)
            s["slots"] = torch.randperm(n_pages * c.page, generator=gen, device="cuda")[:c.T].to(torch.int32)
            if c.T > 4 * c.page:                 # prompts: pages in any order, the tokens of a page side by side
                t = torch.arange(c.T, device="cuda")
                s["slots"] = (torch.randperm(n_pages, generator=gen, device="cuda")[t // c.page] * c.page + t % c.page).to(torch.int32)
            if getattr(c, "skip", False):
                s["slots"][torch.rand(c.T, generator=gen, device="cuda") < 0.02] = -1
    else:
        n_pool = sum(c.pages) + 3
        table = torch.zeros((c.B, c.max_pages), dtype=torch.int32, device="cuda")
        here = torch.arange(c.max_pages, device="cuda")[None] < ints(c.pages)[:, None]
        table[here] = torch.randperm(n_pool, generator=gen, device="cuda").to(torch.int32)[:sum(c.pages)]
        s = dict(k_pool=pool(n_pool), v_pool=pool(n_pool), table=table, lens=ints(c.lens))
        rows = c.T if c.op == "prefill" else c.B
        s["q"] = (normal(rows, c.H, c.d) * 1.5).to(c.st)
        s["o"] = empty(rows, c.H, c.d)
        s["lse"] = torch.empty((rows, c.H), dtype=torch.float32, device="cuda")
        if c.op == "prefill":
            s["cu"] = ints([sum(c.news[:b]) for b in range(c.B + 1)])
    s["c"] = c
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    c = s["c"]
    return (_own if own else _plain)[c.op](c, s)


def _normed_and_turned(c, x, weight, cos, sin):
    x = x.float()
    x = x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.float()
    rot, rest = x[..., :c.rot], x[..., c.rot:]
    if c.layout == "interleaved":
        a, b = rot[..., 0::2], rot[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = rot[..., :c.rot // 2], rot[..., c.rot // 2:]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([y, rest], dim=-1).to(c.st)


def _sines(s):
    angle = s["positions"].double()[:, None, None] * s["freq"]
    return angle.cos().float(), angle.sin().float()


def _norm_rotary_plain(c, s):
    cos, sin = _sines(s)
    s["q_out"].copy_(_normed_and_turned(c, s["q"], s["w_q"], cos, sin))
    s["k_out"].copy_(_normed_and_turned(c, s["k"], s["w_k"], cos, sin))
    return s["q_out"], s["k_out"]


def _append_plain(c, s):
    cos, sin = _sines(s)
    s["q_out"].copy_(_normed_and_turned(c, s["q"], s["w_q"], cos, sin))
    there = s["slots"] >= 0
    slots = s["slots"][there].long()
    s["k_pool"][slots // c.page, :, slots % c.page] = _normed_and_turned(c, s["k"], s["w_k"], cos, sin)[there]
    s["v_pool"][slots // c.page, :, slots % c.page] = s["v"][there]
    return s["q_out"], s["k_pool"], s["v_pool"]


def _cached(c, s, name):
    """The cached rows of every sequence [B, H_kv, tokens of whole table rows, d] as floats."""
    return s[name][s["table"].long()].permute(0, 2, 1, 3, 4).reshape(c.B, c.H_kv, c.max_pages * c.page, c.d).float()


def _attend(c, q, k, v, sees):
    """q [B, H_kv, n, G, d], k and v [B, H_kv, keys, d], sees [B, n, keys] -> o [B, H_kv, n, G, d], lse [B, H_kv, n, G]."""
    B, n, keys = sees.shape
    x = torch.matmul(q.reshape(B, c.H_kv, n * c.group, c.d), k.transpose(-1, -2).contiguous()).mul_(c.scale)
    x = x.reshape(B, c.H_kv, n, c.group, keys).masked_fill_(~sees[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.reshape(B, c.H_kv, n * c.group, keys), v).reshape(B, c.H_kv, n, c.group, c.d)
    return torch.where(total > 0, o / total, 0.0), (total.log() + top)[..., 0]


def _decode_plain(c, s):
    sees = torch.arange(c.max_pages * c.page, device="cuda")[None, None] < s["lens"][:, None, None]
    q = s["q"].float().reshape(c.B, c.H_kv, 1, c.group, c.d)
    there = sees.reshape(c.B, 1, -1, 1)
    o, lse = _attend(c, q, _cached(c, s, "k_pool") * there, _cached(c, s, "v_pool") * there, sees)
    s["o"].copy_(o.reshape(c.B, c.H, c.d))
    s["lse"].copy_(lse.reshape(c.B, c.H))
    return s["o"], s["lse"]


def _prefill_plain(c, s):
    cu, L = s["cu"].long(), s["lens"].long()
    n = max(c.news)
    i = torch.arange(n, device="cuda")
    there = i[None] < (cu[1:] - cu[:-1])[:, None]                            # [B, n]
    rows = torch.where(there, cu[:-1, None] + i, 0)
    t = torch.arange(c.max_pages * c.page, device="cuda")
    sees = (t[None, None] <= (L[:, None] + i)[:, :, None]) & there[:, :, None]
    cached = (t < (L + cu[1:] - cu[:-1])[:, None]).reshape(c.B, 1, -1, 1)
    q = s["q"].float()[rows].reshape(c.B, n, c.H_kv, c.group, c.d).transpose(1, 2)
    o, lse = _attend(c, q, _cached(c, s, "k_pool") * cached, _cached(c, s, "v_pool") * cached, sees)
    s["o"].copy_(o.transpose(1, 2).reshape(c.B, n, c.H, c.d)[there])         # (sequences are packed in their order)
    s["lse"].copy_(lse.transpose(1, 2).reshape(c.B, n, c.H)[there])
    return s["o"], s["lse"]


_plain = {"norm_rotary": _norm_rotary_plain, "append": _append_plain, "decode": _decode_plain, "prefill": _prefill_plain}


# ------------------------------------------------------------------ the framework's calls
def _shape(c, tp, B):
    return tp.TplaHeads(B, c.H, c.H_kv, c.d, c.d, c.page, tp.TPLA_F32 if c.dtype == "f32" else tp.TPLA_BF16, c.scale)


def _layout(c, tp):
    return tp.TPLA_ROTARY_INTERLEAVED if c.layout == "interleaved" else tp.TPLA_ROTARY_HALF


def _norm_rotary_own(c, s):
    import paper_2508_15881_amd as tp
    tp.tpla_norm_rotary_heads(_shape(c, tp, 1), _layout(c, tp), c.rot, s["freq"], 1.0, s["w_q"], s["w_k"], EPS, s["positions"], c.T,
                              s["q"], s["q_out"], s["k"], s["k_out"])
    return s["q_out"], s["k_out"]


def _append_own(c, s):
    import paper_2508_15881_amd as tp
    tp.tpla_append_heads(_shape(c, tp, 1), _layout(c, tp), c.rot, s["freq"], 1.0, s["w_q"], s["w_k"], EPS, s["positions"], c.T,
                         s["q"], s["q_out"], s["k"], s["v"], s["slots"], s["k_pool"], s["v_pool"])
    return s["q_out"], s["k_pool"], s["v_pool"]


def _workspace(s, n_bytes):
    """A program keeps its workspace; one of the same shapes needs the same."""
    if "workspace" not in s:
        s["workspace"] = torch.empty(max(16, n_bytes()), dtype=torch.uint8, device="cuda")
    return s["workspace"], s["workspace"].numel()


def _decode_own(c, s):
    import paper_2508_15881_amd as tp
    shape = _shape(c, tp, c.B)
    ws, n = _workspace(s, lambda: tp.tpla_workspace_bytes_heads(shape, c.max_pages))
    tp.tpla_decode_heads(shape, s["q"], s["k_pool"], s["v_pool"], s["table"], c.max_pages, s["lens"], ws, n, s["o"], shape.dtype, s["lse"])
    return s["o"], s["lse"]


def _prefill_own(c, s):
    import paper_2508_15881_amd as tp
    shape = _shape(c, tp, c.B)
    ws, n = _workspace(s, lambda: tp.tpla_workspace_bytes_prefill_heads(shape, c.T, max(c.news), c.max_pages))
    tp.tpla_prefill_heads(shape, s["q"], s["k_pool"], s["v_pool"], s["table"], c.max_pages, s["lens"], s["cu"], c.T, max(c.news), ws, n,
                          s["o"], shape.dtype, s["lse"])
    return s["o"], s["lse"]


_own = {"norm_rotary": _norm_rotary_own, "append": _append_own, "decode": _decode_own, "prefill": _prefill_own}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = _Case(case)
    if c.op in ("norm_rotary", "append"):
        n = c.T * (c.H + c.H_kv)
        moved = n + (c.T * c.H_kv if c.op == "append" else 0)
        return {"bytes": 2.0 * moved * c.d * c.esz + 8 * c.T + 4 * c.rot, "flops": n * (4.0 * c.d + 3.0 * c.rot)}
    rows = c.T if c.op == "prefill" else c.B
    pairs = sum(n * L + n * (n + 1) // 2 for n, L in zip(c.news, c.lens)) if c.op == "prefill" else sum(c.lens)
    return {"bytes": float(c.esz) * (2 * sum(c.keys) * c.H_kv * c.d + 2 * rows * c.H * c.d) + 4.0 * rows * c.H + 4 * sum(c.pages),
            "flops": 4.0 * pairs * c.H * c.d}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c.op in ("norm_rotary", "append"):
        angle = s["positions"].double()[:, None] * s["freq"]
        z = torch.polar(torch.ones_like(angle), angle)[:, None]

        def of(x, w):
            x = x.double()
            x = x * w.double() * torch.rsqrt(x.square().sum(-1, keepdim=True) / c.d + EPS)
            r = x[..., :c.rot]
            pair = r.unflatten(-1, (c.rot // 2, 2)) if c.layout == "interleaved" else r.unflatten(-1, (2, c.rot // 2)).transpose(-1, -2)
            y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * z)
            y = y if c.layout == "interleaved" else y.transpose(-1, -2)
            return torch.cat([y.flatten(-2), x[..., c.rot:]], -1)

        q, k = of(s["q"], s["w_q"]), of(s["k"], s["w_k"])
        if c.op == "norm_rotary":
            return q, k
        pools = [s["k_pool"].double().transpose(1, 2).flatten(0, 1), s["v_pool"].double().transpose(1, 2).flatten(0, 1)]
        used = torch.nonzero(s["slots"] >= 0)[:, 0]
        for p, x in zip(pools, (k, s["v"].double())):
            p[s["slots"][used].long()] = x[used]
        return (q, *(p.unflatten(0, (-1, c.page)).transpose(1, 2) for p in pools))
    rows = c.T if c.op == "prefill" else c.B
    o = torch.zeros((rows, c.H, c.d), dtype=torch.float64, device="cuda")
    lse = torch.full((rows, c.H), -math.inf, dtype=torch.float64, device="cuda")
    first = 0
    for b in range(c.B):
        n = c.news[b] if c.op == "prefill" else 1
        ids = s["table"][b, :c.pages[b]].long()
        K = s["k_pool"][ids].double().transpose(0, 1).flatten(1, 2)[:, :c.keys[b]]
        V = s["v_pool"][ids].double().transpose(0, 1).flatten(1, 2)[:, :c.keys[b]]
        for h in range(c.H):
            kh, vh = K[h // c.group], V[h // c.group]
            for i0 in range(0, n, 4096):
                i1 = min(n, i0 + 4096)
                x = c.scale * (s["q"][first + i0:first + i1, h].double() @ kh.T)
                if c.op == "prefill":
                    x += torch.full_like(x, -math.inf).triu(c.lens[b] + i0 + 1)
                z = torch.logsumexp(x, -1)
                lse[first + i0:first + i1, h] = z
                o[first + i0:first + i1, h] = torch.exp(x - z[:, None]) @ vh
        first += n
    return o, lse
