"""The operators of a speculative decode step over the sliced latent cache, as cases that can be timed and compared.

A case is a dict of plain values.  Its "op" says which operator one pass runs:

  extend  tpla_extend_sequences: pages for the new tokens of every sequence from a list of free ones, the slot and the
          position of every new token.  row_tokens > 0: a row of that many per sequence (decode, drafts), else packed.
  rotary  tpla_apply_rotary: queries [T, H, d_r], a view into the query projection's [T, H, d_n + d_r], and keys [T, d_r].
  tree    tpla_decode_shards_tree_combine: T drafted tokens per sequence attend to the committed tokens and to the drafts
          that their mask names, over all latent slices; value up-projection and sum over the slices.
  commit  tpla_commit_drafts: the rows of the accepted drafts move behind the committed ones, the lengths grow.

Where `own` is false the plain form of the operator runs: elementary torch operations in 32 bits (angles in 64).
"""
import math

import torch

own = False

D_C, D_R, D_N, D_V = 512, 64, 128, 128
DEFAULTS = dict(H=64, d_c=D_C, g=2, d_r=D_R, d_n=D_N, d_v=D_V, dtype="bf16", page=64)
MOST_SCORES = 2 * 16 * 16 * 64 * 32768           # scores of the largest listed tree case


def listed():
    return [
        # one new token for each of 48 running sequences: all latency
        dict(name="extend_decode", op="extend", B=48, row_tokens=1, min_len=5, max_len=8000, min_add=1, max_add=1),
        # a batch of draft trees of uneven sizes, depths given
        dict(name="extend_drafts", op="extend", B=120, row_tokens=24, min_len=100, max_len=30000, min_add=0, max_add=24, depths=True, page=16),
        # prompts of many lengths admitted at once, packed
        dict(name="extend_prompts", op="extend", B=93, row_tokens=0, min_len=1, max_len=3, min_add=501, max_add=32768),
        # one user's next token
        dict(name="rotary_one", op="rotary", T=1, layout="interleaved", far=120000),
        # the float configuration users check results with, part of the head, halves
        dict(name="rotary_f32_part", op="rotary", T=1537, H=4, d_n=32, d_r=48, rot=32, layout="half", dtype="f32", far=4000),
        # prompts of a prefill batch, far positions, pairs side by side
        dict(name="rotary_prompts", op="rotary", T=20011, layout="interleaved", far=131072, scaled=True),
        # the float configuration: smallest call
        dict(name="tree_f32_tiny", op="tree", B=2, T=5, H=4, d_c=64, d_r=16, d_n=32, d_v=32, dtype="f32", min_len=60, max_len=128, min_draft=3),
        # one user with a wide tree, short context
        dict(name="tree_one_user", op="tree", B=1, T=26, min_len=1237, max_len=1237, min_draft=26),
        # a serving batch: odd lengths, chains of up to 5 with 16 heads on this device: bound by the cache
        dict(name="tree_chain_16_heads", op="tree", B=37, T=5, H=16, min_len=900, max_len=20011, min_draft=1, chain=True),
        # the largest: 16 drafts for each of 16 sequences of 32768 tokens
        dict(name="tree_32k", op="tree", B=16, T=16, min_len=32768, max_len=32768, min_draft=16),
        # two or three accepted of eight
        dict(name="commit_small", op="commit", B=24, T=8, min_len=100, max_len=3000, most=3),
        # long drafts in a large batch over four slices, most of them accepted
        dict(name="commit_large", op="commit", B=240, T=64, g=4, min_len=33, max_len=2000, most=60),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["extend", "rotary", "rotary", "tree", "tree", "tree", "tree", "commit"])
    if op == "extend":
        rows = rng.choice([0, 1, 3, 8, 17, 64])
        c = dict(op=op, B=_log_uniform(rng, 1, 128), row_tokens=rows, page=rng.choice([16, 32, 64, 64, 128]), max_len=_log_uniform(rng, 10, 30000))
        c["min_len"] = max(1, c["max_len"] // rng.randint(1, 32))
        c["max_add"] = rows if rows else _log_uniform(rng, 20, 16000)
        c["min_add"] = max(1, c["max_add"] // rng.randint(1, 8))
        c["depths"] = bool(rows > 1 and rng.random() < 0.5)
        return c
    if op == "rotary":
        d_r = rng.choice([16, 32, 64, 64, 64, 128])
        return dict(op=op, T=_log_uniform(rng, 1, 10000), H=rng.choice([1, 5, 16, 32, 64]), d_r=d_r, rot=rng.choice([d_r, d_r, d_r // 2, d_r - 4]),
                    layout=rng.choice(["interleaved", "half"]), dtype=rng.choice(["bf16", "bf16", "f32"]), far=_log_uniform(rng, 100, 1000000),
                    scaled=rng.random() < 0.5)
    if op == "commit":
        c = dict(op=op, B=_log_uniform(rng, 1, 200), T=rng.randint(1, 64), H=16, g=rng.choice([1, 2, 4]), page=rng.choice([16, 64, 64]), max_len=_log_uniform(rng, 10, 2000))
        c["min_len"], c["most"] = max(1, c["max_len"] // 8), rng.randint(1, c["T"])
        return c
    if rng.random() < 0.15:
        hi = _log_uniform(rng, 1, 1000)
        T = rng.randint(1, 9)
        return dict(op=op, B=rng.randint(1, 5), T=T, H=rng.choice([1, 4, 7]), d_c=64, d_r=16, d_n=32, d_v=32, dtype="f32", g=rng.choice([1, 2]),
                    min_len=max(1, hi // 3), max_len=hi, min_draft=1, page=rng.choice([16, 64]))
    hi = _log_uniform(rng, 1, 32768)
    c = dict(op=op, B=_log_uniform(rng, 1, 64), T=_log_uniform(rng, 1, 64), H=rng.choice([8, 16, 32, 64, 64, 128]), g=rng.choice([1, 2, 2, 2, 4]),
             page=rng.choice([16, 64, 64, 64, 128]), min_len=max(1, hi // rng.randint(1, 8)), max_len=hi, chain=rng.random() < 0.4)
    c["min_draft"] = rng.randint(1, c["T"])
    while c["B"] > 1 and 4 * c["g"] * c["B"] * c["T"] * c["H"] * (hi + c["T"]) > MOST_SCORES:
        c["B"] = c["B"] * 2 // 3
    while 4 * c["g"] * c["B"] * c["T"] * c["H"] * (hi + c["T"]) > MOST_SCORES:
        c["T"] = c["T"] * 2 // 3
    c["min_draft"] = min(c["min_draft"], c["T"])
    return c


# ------------------------------------------------------------------ inputs
class _Case:
    def __init__(self, case):
        for k, v in {**DEFAULTS, **case}.items():
            setattr(self, k, v)
        self.dl = self.d_c // self.g
        self.st = torch.float32 if self.dtype == "f32" else torch.bfloat16
        self.esz = 4 if self.dtype == "f32" else 2
        self.scale = 1.0 / math.sqrt(self.d_n + self.d_r)
        if self.op != "rotary":
            self.lens = _spread(self.min_len, self.max_len, self.B)
        if self.op == "extend":
            self.adds = _spread(self.min_add, self.max_add, self.B)[::-1]
            self.n_tokens = self.B * self.row_tokens if self.row_tokens else sum(self.adds)
            self.max_pages = max(-(-(a + b) // self.page) for a, b in zip(self.lens, self.adds)) + 3
        if self.op == "tree":
            self.drafts = _spread(self.min_draft, self.T, self.B)
        if self.op == "commit":
            self.takes = _spread(1, min(self.most, self.T), self.B)
            self.drafts = [self.T] * self.B
        if self.op in ("tree", "commit"):
            self.pages = [-(-(a + b) // self.page) for a, b in zip(self.lens, self.drafts)]
            self.max_pages = max(self.pages)
        if self.op == "rotary":
            self.rot = getattr(self, "rot", self.d_r)


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly over the logarithm (0 counts as below 1), in an order that mixes them."""
    v = [min(hi, max(lo, int((lo + 0.5) * ((hi + 0.5) / (lo + 0.5)) ** (i / max(1, n - 1))))) for i in range(n - 1)] + [hi]
    step = next(s for s in range(n // 2 + 1, 2 * n + 2) if math.gcd(s, n) == 1)
    return [v[(i * step + n - 1) % n] for i in range(n)]


def _frequencies(c):
    """Radians per position of each pair, 64 bits.  scaled: contexts 32 times as long as the first 4096 positions, the fast pairs as they were."""
    j = torch.arange(c.rot // 2, dtype=torch.float64)
    f = 10000.0 ** (-2.0 * j / c.rot)
    if getattr(c, "scaled", False):
        at = lambda turns: c.rot * math.log(4096 / (2 * math.pi * turns)) / (2 * math.log(10000.0))  # noqa: E731
        low, high = max(0, math.floor(at(32.0))), min(c.rot - 1, math.ceil(at(1.0)))
        slow = ((j - low) / max(high - low, 1e-3)).clamp(0, 1)
        f = f * (1 - slow) + f / 32.0 * slow
    return f.cuda()


def prepare(case, seed):
    c = _Case(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    normal = lambda *n: torch.randn(n, generator=gen, device="cuda")  # noqa: E731
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    if c.op == "extend":
        held = [-(-n // c.page) for n in c.lens]
        n_pool = sum(-(-(a + b) // c.page) for a, b in zip(c.lens, c.adds)) + 17
        order = torch.randperm(n_pool, generator=gen, device="cuda").to(torch.int32)
        table = torch.zeros((c.B, c.max_pages), dtype=torch.int32, device="cuda")
        here = torch.arange(c.max_pages, device="cuda")[None] < ints(held)[:, None]
        table[here] = order[:sum(held)]
        s = dict(lens=ints(c.lens), adds=ints(c.adds), held=ints(held), table=table, free=order[sum(held):].clone(), depths=None)
        if getattr(c, "depths", False):
            s["depths"] = torch.minimum(torch.randint(0, 6, (c.B, c.row_tokens), generator=gen, device="cuda"),
                                        torch.arange(c.row_tokens, device="cuda")[None]).to(torch.int32)
        for k, n in (("held_out", c.B), ("cu", c.B + 1), ("slots", c.n_tokens), ("positions", c.n_tokens), ("counts", 2)):
            s[k] = torch.zeros(n, dtype=torch.int32, device="cuda")
    elif c.op == "rotary":
        q = normal(c.T, c.H, c.d_n + c.d_r).to(c.st)
        s = dict(q=q[:, :, c.d_n:], k=normal(c.T, c.d_r).to(c.st), freq=_frequencies(c),
                 positions=torch.randint(0, c.far, (c.T,), generator=gen, device="cuda").to(torch.int32),
                 q_out=torch.empty((c.T, c.H, c.d_r), dtype=c.st, device="cuda"), k_out=torch.empty((c.T, c.d_r), dtype=c.st, device="cuda"))
    else:
        n_pool = sum(c.pages) + 3
        pools = torch.empty((c.g, n_pool, c.page, c.dl + c.d_r), dtype=c.st, device="cuda")
        for i in range(c.g):
            pools[i] = normal(n_pool, c.page, c.dl + c.d_r).to(c.st)
        table = torch.zeros((c.B, c.max_pages), dtype=torch.int32, device="cuda")
        here = torch.arange(c.max_pages, device="cuda")[None] < ints(c.pages)[:, None]
        table[here] = torch.randperm(n_pool, generator=gen, device="cuda").to(torch.int32)[:sum(c.pages)]
        s = dict(pools=pools, table=table, lens=ints(c.lens))
        if c.op == "tree":
            t = torch.arange(c.T, device="cuda")
            if getattr(c, "chain", False):
                parent = (t - 1).expand(c.B, c.T)
            else:                                 # each draft continues one of the seven before it, or the committed tokens
                parent = (t - torch.randint(1, 8, (c.B, c.T), generator=gen, device="cuda")).clamp(min=-1)
            sees = torch.eye(c.T, dtype=torch.bool, device="cuda").expand(c.B, c.T, c.T).clone()
            for j in range(1, c.T):               # a draft sees what its parent sees
                p = parent[:, j]
                sees[:, j] |= sees[torch.arange(c.B, device="cuda"), p.clamp(min=0)] & (p >= 0)[:, None]
            s["mask"] = (sees.to(torch.int64) << t.to(torch.int64)[None, None]).sum(2)      # bit j: draft j is seen
            s["drafts"] = ints(c.drafts)
            s["q_lat"] = (normal(c.g, c.B, c.T, c.H, c.dl) * 0.35).to(c.st)
            s["q_pe"] = normal(c.B, c.T, c.H, c.d_r).to(c.st)
            s["W"] = (normal(c.H, c.d_c, c.d_v) * 0.02).to(c.st)
            s["o"] = torch.empty((c.B, c.T, c.H, c.d_v), dtype=c.st, device="cuda")
            s["o_lat"] = torch.empty((c.g, c.B, c.T, c.H, c.dl), dtype=torch.float32, device="cuda")
            s["lse"] = torch.empty((c.g, c.B, c.T, c.H), dtype=torch.float32, device="cuda")
        else:
            key = torch.rand((c.B, c.T), generator=gen, device="cuda")
            kept = key.argsort(1).argsort(1) < ints(c.takes)[:, None]        # a random subset of each sequence's drafts
            s["accepted"] = torch.where(kept, 0, c.T).add(torch.arange(c.T, device="cuda")[None]).argsort(1).to(torch.int32)
            s["n_accepted"] = ints(c.takes)
            s["new_lens"] = torch.zeros(c.B, dtype=torch.int32, device="cuda")
    s["c"] = c
    return s


# ------------------------------------------------------------------ one pass
def run(s):
    c = s["c"]
    return (_own if own else _plain)[c.op](c, s)


def _rows_of(c, table, tokens):
    """Pool rows of tokens [B, n] (counted in their sequences)."""
    page = (tokens // c.page).clamp(0, table.shape[1] - 1)
    return torch.gather(table.long(), 1, page) * c.page + tokens % c.page


def _extend_plain(c, s):
    L, n, held, free = s["lens"].long(), s["adds"].long(), s["held"].long(), s["free"]
    need = (torch.clamp((L + n + c.page - 1) // c.page, max=c.max_pages) - held).clamp(min=0)
    first = need.cumsum(0) - need
    given = torch.minimum(need, (free.numel() - first).clamp(min=0))
    k = torch.arange(c.max_pages, device="cuda")[None] - held[:, None]
    new = (k >= 0) & (k < given[:, None])
    s["table"].copy_(torch.where(new, free[(first[:, None] + k).clamp(0, free.numel() - 1)], s["table"]))
    s["held_out"].copy_(held + given)
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), n.cumsum(0)])
    s["cu"].copy_(cu)
    at = torch.arange(c.n_tokens, device="cuda")
    if c.row_tokens:
        b, i = at // c.row_tokens, at % c.row_tokens
        there = i < n[b]
    else:
        b = torch.searchsorted(cu, at, right=True) - 1
        i = at - cu[b]
        there = at >= 0
    t = L[b] + i
    page = t // c.page
    there = there & (page < (held + given)[b])
    row = s["table"].long()[b, page.clamp(max=c.max_pages - 1)] * c.page + t % c.page
    s["slots"].copy_(torch.where(there, row, -1))
    depth = i if s["depths"] is None else s["depths"].long().reshape(-1)
    s["positions"].copy_(torch.where(i < n[b], L[b] + depth, 0))
    s["counts"].copy_(torch.stack([given.sum(), (need - given).sum()]))
    return {k: s[k] for k in ("table", "held_out", "cu", "slots", "positions", "counts")}


def _turned(c, x, cos, sin):
    x = x.float()
    rot, rest = x[..., :c.rot], x[..., c.rot:]
    if c.layout == "interleaved":
        a, b = rot[..., 0::2], rot[..., 1::2]
        y = torch.stack([a * cos - b * sin, a * sin + b * cos], dim=-1).flatten(-2)
    else:
        a, b = rot[..., :c.rot // 2], rot[..., c.rot // 2:]
        y = torch.cat([a * cos - b * sin, a * sin + b * cos], dim=-1)
    return torch.cat([y, rest], dim=-1).to(c.st)


def _rotary_plain(c, s):
    angle = s["positions"].double()[:, None] * s["freq"][None]
    cos, sin = angle.cos().float(), angle.sin().float()
    s["q_out"].copy_(_turned(c, s["q"], cos[:, None], sin[:, None]))
    s["k_out"].copy_(_turned(c, s["k"], cos, sin))
    return s["q_out"], s["k_out"]


def _tree_plain(c, s):
    n_keys = max(a + b for a, b in zip(c.lens, c.drafts))
    t = torch.arange(n_keys, device="cuda")[None].expand(c.B, n_keys)
    L = s["lens"].long()[:, None]
    there = t < L + s["drafts"].long()[:, None]
    rows = _rows_of(c, s["table"], torch.where(there, t, 0))
    keys = s["pools"].reshape(c.g, -1, c.dl + c.d_r)[:, rows].float() * there[None, :, :, None]      # [g, B, keys, dl + d_r]
    q = torch.cat([s["q_lat"], s["q_pe"][None].expand(c.g, -1, -1, -1, -1)], dim=-1).float().reshape(c.g, c.B, c.T * c.H, -1)
    bit = (s["mask"][:, :, None] >> (t - L).clamp(0, 63)[:, None]) & 1
    sees = (t < L)[:, None] | ((bit == 1) & there[:, None])                                          # [B, T, keys]
    sees = sees & (torch.arange(c.T, device="cuda")[None, :, None] < s["drafts"].long()[:, None, None])
    scores = torch.matmul(q, keys.transpose(-1, -2)) * c.scale
    scores = scores.reshape(c.g, c.B, c.T, c.H, n_keys).masked_fill_(~sees[None, :, :, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    lat = torch.matmul(p.reshape(c.g, c.B, c.T * c.H, n_keys), keys[..., :c.dl]).reshape(c.g, c.B, c.T, c.H, c.dl)
    lat = torch.where(total > 0, lat / total, 0.0)
    s["lse"].copy_((total.log() + top)[..., 0])
    o = torch.matmul(lat.permute(3, 1, 2, 0, 4).reshape(c.H, c.B * c.T, c.d_c), s["W"].float())       # [H, B T, d_v]
    s["o"].copy_(o.reshape(c.H, c.B, c.T, c.d_v).permute(1, 2, 0, 3))
    return s["o"], s["lse"]


def _commit_plain(c, s):
    k = torch.arange(c.T, device="cuda")[None].expand(c.B, c.T)
    moves = k < s["n_accepted"][:, None]
    L = s["lens"].long()[:, None]
    src = _rows_of(c, s["table"], L + s["accepted"].long().clamp(0, c.T - 1))[moves]
    dst = _rows_of(c, s["table"], L + k)[moves]
    flat = s["pools"].reshape(c.g, -1, c.dl + c.d_r)
    flat[:, dst] = flat[:, src]
    s["new_lens"].copy_(s["lens"] + s["n_accepted"])
    return s["pools"], s["new_lens"]


_plain = {"extend": _extend_plain, "rotary": _rotary_plain, "tree": _tree_plain, "commit": _commit_plain}


# ------------------------------------------------------------------ the framework's calls
def _shape(c, tp, B):
    return tp.TplaShape(B, c.H, c.d_c, c.g, c.d_r, c.d_n, c.d_v, c.page, tp.TPLA_F32 if c.dtype == "f32" else tp.TPLA_BF16, c.scale)


def _extend_own(c, s):
    import paper_2508_15881_amd as tp
    tp.tpla_extend_sequences(_shape(c, tp, c.B), s["lens"], s["adds"], c.row_tokens, s["depths"], s["free"], s["free"].numel(), s["held"],
                             s["held_out"], s["table"], c.max_pages, s["cu"], s["slots"], s["positions"], c.n_tokens, s["counts"])
    return {k: s[k] for k in ("table", "held_out", "cu", "slots", "positions", "counts")}


def _rotary_own(c, s):
    import paper_2508_15881_amd as tp
    tp.tpla_apply_rotary(_shape(c, tp, 1), tp.TPLA_ROTARY_INTERLEAVED if c.layout == "interleaved" else tp.TPLA_ROTARY_HALF, 0, c.rot, s["freq"], 1.0,
                         s["positions"], c.T, s["q"], s["q_out"], s["k"], s["k_out"])
    return s["q_out"], s["k_out"]


def _tree_own(c, s):
    import paper_2508_15881_amd as tp
    shape = _shape(c, tp, c.B)
    if "workspace" not in s:
        s["workspace"] = torch.empty(tp.tpla_workspace_bytes_tree(shape, c.T, c.max_pages), dtype=torch.uint8, device="cuda")
    tp.tpla_decode_shards_tree_combine(shape, c.T, s["q_lat"], s["q_pe"], [s["pools"][i] for i in range(c.g)], s["table"], c.max_pages, s["lens"],
                                       s["drafts"], s["mask"], s["workspace"], s["workspace"].numel(), s["W"], s["o"], shape.dtype, s["o_lat"], s["lse"])
    return s["o"], s["lse"]


def _commit_own(c, s):
    import paper_2508_15881_amd as tp
    tp.tpla_commit_drafts(_shape(c, tp, c.B), c.T, s["accepted"], s["n_accepted"], s["lens"], s["table"], c.max_pages,
                          [s["pools"][i] for i in range(c.g)], s["new_lens"])
    return s["pools"], s["new_lens"]


_own = {"extend": _extend_own, "rotary": _rotary_own, "tree": _tree_own, "commit": _commit_own}


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c = _Case(case)
    if c.op == "extend":
        new = sum(-(-(a + b) // c.page) - -(-a // c.page) for a, b in zip(c.lens, c.adds))
        return {"bytes": 4.0 * (5 * c.B + 2 * new + 2 * c.n_tokens), "flops": 0.0}
    if c.op == "rotary":
        n = c.T * (c.H + 1)
        return {"bytes": 2.0 * n * c.d_r * c.esz + 4 * c.T + 8 * c.rot // 2, "flops": 3.0 * n * c.rot}
    if c.op == "commit":
        return {"bytes": 2.0 * c.g * sum(c.takes) * (c.dl + c.d_r) * c.esz + 4 * (sum(c.takes) + 3 * c.B), "flops": 0.0}
    keys = sum(a + b for a, b in zip(c.lens, c.drafts))
    pairs = sum((a + b) * b for a, b in zip(c.lens, c.drafts)) * c.H
    rows = sum(c.drafts) * c.H
    return {"bytes": float(c.esz) * (c.g * keys * (c.dl + c.d_r) + rows * (c.d_c + c.d_r) + c.H * c.d_c * c.d_v + c.B * c.T * c.H * c.d_v)
            + 4.0 * c.g * c.B * c.T * c.H + 8 * c.B * c.T,
            "flops": 2.0 * c.g * pairs * (2 * c.dl + c.d_r) + 2.0 * rows * c.d_c * c.d_v}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c.op in ("extend", "commit"):
        return None                              # whole numbers and moved rows: nothing is rounded
    if c.op == "rotary":
        angle = s["positions"].double()[:, None] * s["freq"]
        z = torch.polar(torch.ones_like(angle), angle)

        def turn(x, by):
            x = x.double()
            r = x[..., :c.rot]
            pair = r.unflatten(-1, (c.rot // 2, 2)) if c.layout == "interleaved" else r.unflatten(-1, (2, c.rot // 2)).transpose(-1, -2)
            y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * by)
            y = y if c.layout == "interleaved" else y.transpose(-1, -2)
            return torch.cat([y.flatten(-2), x[..., c.rot:]], -1)

        return turn(s["q"], z[:, None]), turn(s["k"], z)
    W = s["W"].double()
    o = torch.zeros((c.B, c.T, c.H, c.d_v), dtype=torch.float64, device="cuda")
    lse = torch.full((c.g, c.B, c.T, c.H), -math.inf, dtype=torch.float64, device="cuda")
    for b in range(c.B):
        L, n = c.lens[b], c.drafts[b]
        ids = s["table"][b].tolist()
        pages = [s["pools"][:, p] for p in ids[:c.pages[b]]]
        rows = torch.cat(pages, dim=1)[:, :L + n].double()
        words = [int(v) for v in s["mask"][b].tolist()]
        add = torch.zeros((n, L + n), dtype=torch.float64)
        for t in range(n):
            add[t, L:] = torch.tensor([0.0 if (words[t] >> j) & 1 else -math.inf for j in range(n)], dtype=torch.float64)
        add = add.cuda()
        for i in range(c.g):
            v = rows[i, :, :c.dl]
            for h0 in range(0, c.H, 16):
                hs = slice(h0, min(c.H, h0 + 16))
                x = s["q_lat"][i, b, :n, hs].double() @ v.T + s["q_pe"][b, :n, hs].double() @ rows[i, :, c.dl:].T
                x = x * c.scale + add[:, None]
                z = torch.logsumexp(x, -1)
                lse[i, b, :n, hs] = z
                lat = torch.exp(x - z[..., None]) @ v
                o[b, :n, hs] += torch.matmul(lat.transpose(0, 1), W[hs, i * c.dl:(i + 1) * c.dl]).transpose(0, 1)
    return o, lse
