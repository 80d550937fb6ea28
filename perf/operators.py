"""Operators around a paged key-value cache, as timed cases: what they compute in plain torch, and the library's calls.

Four kinds, each one entry point of `binding`:

  qk_fwd   RMS norm of every query and key head and the rotation by the token's position, one pass (training, prompts)
  qk_bwd   its gradient: queries, keys and the two norm weights
  append   the same on the way into a paged cache: queries beside it, keys and values into the pages (bf16, or e4m3 with a scale a KV head)
  attn     a block of new tokens, or one, against the pages of its sequence

`own` says which of the two `run` takes.  Sizes are those of the workloads in `synth`, of the tests and of the benchmark (heads 32/32, 32/8 and
28/4 of 128, 14/2, 16/2 and 4/4 of 64 and 128; blocks of 4 and 32; prompts of 391 to 8192 tokens; packed batches of 64 k tokens) and lengths around
them; queries, keys and values are N(0, 1) as there.
"""
import math
import random

import torch

own = False

BF16, F32, F64, I32, U8, E4M3 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.uint8, torch.float8_e4m3fn
DEV = "cuda:0"
EPS = 1e-6
LARGEST = 448.0               # of e4m3


# --------------------------------------------------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------------------------------------------------
def _qk(kind, T, seq, Hq, Hkv, d, rot, pairs, norm):
    """T tokens, whose positions start again every `seq`; `rot` entries of a head are rotated (0: none)."""
    return dict(kind=kind, T=T, seq=seq, Hq=Hq, Hkv=Hkv, d=d, rot=rot, pairs=pairs, norm=norm)


def _append(B, lo, hi, before, Hq, Hkv, d, rot, pairs, norm, page, e4m3, padded=0):
    """B sequences that bring lo .. hi tokens each, behind up to `before` tokens that they have; `padded`: tokens without a slot behind them."""
    return dict(kind="append", B=B, lo=lo, hi=hi, before=before, Hq=Hq, Hkv=Hkv, d=d, rot=rot, pairs=pairs, norm=norm, page=page, e4m3=e4m3, padded=padded)


def _attn(B, Lq, lo, hi, Hq, Hkv, d, page, e4m3, bs=0, ragged=False):
    """B sequences of lo .. hi cached tokens, the last Lq of which ask (ragged: 0 to Lq of them); bs: block size of the block-causal mask (0: none)."""
    return dict(kind="attn", B=B, Lq=Lq, lo=lo, hi=hi, Hq=Hq, Hkv=Hkv, d=d, page=page, e4m3=e4m3, bs=bs, ragged=ragged)


def listed():
    return [
        # one denoising step of the benchmark's default rollout (8 sequences, blocks of 32): a few microseconds, launch and latency
        dict(_qk("qk_fwd", 256, 32, 32, 32, 128, 128, False, False), name="qk_fwd_block"),
        # the training forward of a grouped-query model with normalised heads: 32 sequences of 4096 tokens
        dict(_qk("qk_fwd", 131072, 4096, 32, 8, 128, 128, False, True), name="qk_fwd_train"),
        # a micro-batch of a small model, odd length
        dict(_qk("qk_bwd", 333, 111, 14, 2, 64, 64, False, True), name="qk_bwd_small"),
        # half of every head rotated, neighbours paired, an odd number of tokens
        dict(_qk("qk_bwd", 12289, 12289, 28, 4, 128, 64, True, True), name="qk_bwd_partial"),
        # the actor update's packed batch: 64 k tokens, multi-head, normalised
        dict(_qk("qk_bwd", 65536, 512, 32, 32, 128, 128, False, True), name="qk_bwd_packed"),
        # one token of each of 59 sequences, padded to the 64 that the loop was recorded with
        dict(_append(59, 1, 1, 4095, 32, 8, 128, 128, False, True, 64, False, padded=5), name="append_tokens"),
        # a block of 32 of each of 8 sequences into an 8-bit cache
        dict(_append(8, 32, 32, 768, 32, 32, 128, 128, False, False, 32, True), name="append_block_e4m3"),
        # prompts of a batch job, packed without padding, small pages
        dict(_append(32, 391, 1536, 0, 28, 4, 128, 128, False, False, 16, False), name="append_prompts"),
        # single tokens of a small model: latency
        dict(_attn(3, 1, 1, 400, 14, 2, 64, 16, False), name="attn_token_small"),
        # one token of one long conversation: too few heads to fill the chip without a split
        dict(_attn(1, 1, 65536, 65536, 32, 8, 128, 64, False), name="attn_token_long"),
        # a block-diffusion model's blocks of 4 in 64 sequences of unequal lengths
        dict(_attn(64, 4, 2048, 4096, 32, 8, 128, 64, False, bs=4), name="attn_block_causal"),
        # blocks of up to 32 against an 8-bit cache, seven query heads a KV head: 224 rows share a head's keys
        dict(_attn(32, 32, 391, 1024, 28, 4, 128, 128, True, ragged=True), name="attn_block_e4m3"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_HEADS = [(4, 4, 64), (14, 2, 64), (16, 2, 128), (32, 32, 128), (28, 4, 128), (32, 8, 128)]


def draw(rng):
    kind = rng.choice(["qk_fwd", "qk_bwd", "append", "attn", "attn"])
    Hq, Hkv, d = rng.choice(_HEADS)
    rot, pairs, norm = rng.choice([d, d, d // 2, 0]), rng.random() < 0.3, rng.random() < 0.6
    if not rot:
        norm = True
    page, e4m3 = rng.choice([16, 32, 64, 64, 128, 256]), rng.random() < 0.4
    most = 65536 * 64 * 128 // ((Hq + Hkv) * d)          # tokens that bring as many entries as the largest listed case
    if kind in ("qk_fwd", "qk_bwd"):
        T = _log(rng, 1, min(most, 131072))
        return _qk(kind, T, min(T, _log(rng, 1, 8192)), Hq, Hkv, d, rot, pairs, norm)
    if kind == "append":
        B = _log(rng, 1, 128)
        hi = rng.choice([1, 4, 32, _log(rng, 2, max(2, min(8192, most // (4 * B))))])
        lo = hi if hi in (1, 4, 32) else _log(rng, 1, hi)
        return _append(B, lo, hi, _log(rng, 1, 8192), Hq, Hkv, d, rot, pairs, norm, page, e4m3, padded=rng.choice([0, 0, 1, 7]))
    B = _log(rng, 1, 128)
    hi = _log(rng, 2, max(4, min(65536, (1 << 28) // (B * Hkv * d))))
    Lq = min(rng.choice([1, 1, 4, 8, 17, 32, 32]), hi)
    lo = _log(rng, max(1, Lq), hi) if hi > Lq else hi
    return _attn(B, Lq, lo, hi, Hq, Hkv, d, page, e4m3, bs=rng.choice([0, 0, 1, 4, 32]), ragged=Lq > 1 and rng.random() < 0.3)


def _lengths(case, lo, hi):
    """The case's own lengths, so that its work is the case's; their order in the batch is the seed's."""
    rng = random.Random(1000003 * case["B"] + 1009 * lo + hi)
    return [hi] + [rng.randint(lo, hi) for _ in range(case["B"] - 1)]


# --------------------------------------------------------------------------------------------------------------------
# what a user has in hand before the call
# --------------------------------------------------------------------------------------------------------------------
class _Draw:
    """Seeded draws on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.host = torch.Generator().manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=BF16)

    def weight(self, d):
        return (1.0 + 0.2 * torch.randn(d, generator=self.g, device=DEV)).to(BF16)

    def scales(self, n):
        """One scale a KV head that lets N(0, 1) use most of what 8 bits have."""
        return 0.01 + 0.01 * torch.rand(n, generator=self.g, device=DEV)

    def pages(self, shape, e4m3):
        return (self.normal(*shape) * 64.0).clamp_(-LARGEST, LARGEST).to(E4M3) if e4m3 else self.normal(*shape)

    def order(self, n):
        return torch.randperm(n, generator=self.host)


def _rope_table(n, rot):
    """Row p: the cosines, then the sines, of p / 10000^(2 i / rot), from angles in 64 bits."""
    freq = 10000.0 ** (-torch.arange(0, rot, 2, device=DEV, dtype=F64) / rot)
    angle = torch.arange(n, device=DEV, dtype=F64)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1).to(F32)


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, _Draw(seed))


def _heads(c, r, T, v):
    """Queries and keys (and values) as the projection leaves them: side by side in one buffer."""
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    x = r.normal(T, Hq + (2 if v else 1) * Hkv, d)
    s = dict(kind=c["kind"], case=c, q=x[:, :Hq], k=x[:, Hq:Hq + Hkv], v=x[:, Hq + Hkv:])
    s["qw"], s["kw"] = (r.weight(d), r.weight(d)) if c["norm"] else (None, None)
    return s


def _prepare_qk(c, r):
    T = c["T"]
    s = _heads(c, r, T, False)
    s["pos"] = (torch.arange(T, device=DEV) % c["seq"]).to(I32)
    s["rope"] = _rope_table(c["seq"], c["rot"]) if c["rot"] else None
    for x in ("q", "k"):
        s[x + "_out"] = torch.zeros_like(s[x], memory_format=torch.contiguous_format)
    if c["kind"] == "qk_bwd":
        for x in ("q", "k"):
            s["d_" + x + "_out"] = r.normal(*s[x].shape)
        s["dqw"], s["dkw"] = (torch.zeros(c["d"], dtype=F32, device=DEV) for _ in range(2))
    return s


def _page_tables(r, counts, n_spare):
    """A table row a sequence, of pages in random order; the pool has some that nobody owns."""
    n = sum(counts) + n_spare
    table = torch.zeros((len(counts), max(max(counts), 1)), dtype=I32)
    own_pages, at = r.order(n)[:sum(counts)].to(I32), 0
    for b, m in enumerate(counts):
        table[b, :m] = own_pages[at:at + m]
        at += m
    return n, table


def _prepare_append(c, r):
    B, page = c["B"], c["page"]
    order = r.order(B).tolist()
    new = [_lengths(c, c["lo"], c["hi"])[i] for i in order]
    before = [_lengths(c, 0, c["before"])[i] for i in order]
    n_pages, table = _page_tables(r, [-(-(m + n) // page) for m, n in zip(before, new)], 3)
    new, before = torch.tensor(new), torch.tensor(before)
    first = torch.cumsum(new, 0) - new
    seq = torch.repeat_interleave(torch.arange(B), new)
    pos = before[seq] + torch.arange(int(new.sum())) - first[seq]
    slots = table[seq, pos // page].to(torch.int64) * page + pos % page
    none = torch.zeros(c["padded"], dtype=torch.int64)
    s = _heads(c, r, int(new.sum()) + c["padded"], True)
    s["pos"], s["slots"] = (torch.cat([a, b]).to(I32).to(DEV) for a, b in ((pos, none), (slots, none - 1)))
    s["rope"] = _rope_table(c["before"] + c["hi"], c["rot"]) if c["rot"] else None
    s["q_out"] = torch.zeros_like(s["q"], memory_format=torch.contiguous_format)
    s["cache_k"], s["cache_v"] = (r.pages((n_pages, c["Hkv"], page, c["d"]), c["e4m3"]) for _ in range(2))
    s["ks"], s["vs"] = (r.scales(c["Hkv"]), r.scales(c["Hkv"])) if c["e4m3"] else (None, None)
    return s


def _prepare_attn(c, r):
    B, Lq, page = c["B"], c["Lq"], c["page"]
    order = r.order(B).tolist()
    lens = [_lengths(c, c["lo"], c["hi"])[i] for i in order]
    n_pages, table = _page_tables(r, [-(-n // page) for n in lens], 3)
    s = dict(kind="attn", case=c, q=r.normal(B, Lq, c["Hq"], c["d"]), table=table.to(DEV), lens=torch.tensor(lens, dtype=I32, device=DEV), longest=max(lens))
    s["asks"] = torch.tensor([_lengths(c, 0, Lq)[i] for i in order], dtype=I32, device=DEV) if c["ragged"] else None
    s["cache_k"], s["cache_v"] = (r.pages((n_pages, c["Hkv"], page, c["d"]), c["e4m3"]) for _ in range(2))
    s["ks"], s["vs"] = (r.scales(c["Hkv"]), r.scales(c["Hkv"])) if c["e4m3"] else (None, None)
    # rows behind a sequence's last one stay as they are
    s["out"], s["lse"] = torch.zeros_like(s["q"]), torch.zeros((B, c["Hq"], Lq), dtype=F32, device=DEV)
    return s


_PREPARE = dict(qk_fwd=_prepare_qk, qk_bwd=_prepare_qk, append=_prepare_append, attn=_prepare_attn)


# --------------------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_OWN if own else _PLAIN)[state["kind"]](state)


# ---- in plain torch -------------------------------------------------------------------------------------------------
def _norm(x, w):
    return x if w is None else x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()


def _angles(s):
    """Cosines and sines of every token, [T, 1, rot / 2]."""
    rows = s["rope"][s["pos"].long()][:, None]
    return rows[..., :rows.shape[-1] // 2], rows[..., rows.shape[-1] // 2:]


def _rotate(s, x, sign):
    """x [T, H, d] in 32 bits, rotated by sign times the token's angles."""
    rot, pairs = s["case"]["rot"], s["case"]["pairs"]
    if not rot:
        return x
    cos, sin = _angles(s)
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if pairs else (x[..., :rot // 2], x[..., rot // 2:rot])
    y0, y1 = a * cos - sign * b * sin, b * cos + sign * a * sin
    y = torch.stack([y0, y1], dim=-1).flatten(-2) if pairs else torch.cat([y0, y1], dim=-1)
    return torch.cat([y, x[..., rot:]], dim=-1)


def _plain_qk(s):
    return dict(q=_rotate(s, _norm(s["q"].float(), s["qw"]), 1.0).to(BF16), k=_rotate(s, _norm(s["k"].float(), s["kw"]), 1.0).to(BF16))


def _plain_grad(s, name):
    dz, w = _rotate(s, s["d_" + name + "_out"].float(), -1.0), s[name + "w"]
    if w is None:
        return dz.to(BF16), None
    x = s[name].float()
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS)
    n, g = x * r, dz * w.float()
    return (r * (g - n * (g * n).mean(-1, keepdim=True))).to(BF16), (dz * n).double().sum((0, 1)).float()


def _plain_qk_bwd(s):
    (dq, dqw), (dk, dkw) = _plain_grad(s, "q"), _plain_grad(s, "k")
    got = dict(d_q=dq, d_k=dk)
    return got if dqw is None else dict(got, d_qw=dqw, d_kw=dkw)


def _bits(x):
    """The 8- or 16-bit patterns of a cache: what indexing works on for every type."""
    return x.view(U8 if x.dtype == E4M3 else torch.int16)


def _plain_append(s):
    c, slots = s["case"], s["slots"].long()
    k, v = _rotate(s, _norm(s["k"].float(), s["kw"]), 1.0), s["v"].float()
    live = slots >= 0
    if c["padded"]:
        slots, k, v = slots[live], k[live], v[live]
    for cache, x, scale in ((s["cache_k"], k, s["ks"]), (s["cache_v"], v, s["vs"])):
        x = x.to(BF16) if scale is None else (x / scale[:, None]).clamp(-LARGEST, LARGEST).to(E4M3)
        _bits(cache)[slots // c["page"], :, slots % c["page"]] = _bits(x)
    return dict(q=_rotate(s, _norm(s["q"].float(), s["qw"]), 1.0).to(BF16), cache_k=s["cache_k"], cache_v=s["cache_v"])


def _gathered(s, cache, scale):
    """[B, Hkv, longest, d] in 32 bits; rows behind a sequence's end are whatever the pages hold there."""
    x = _bits(cache)[s["table"].long()].view(cache.dtype).float()              # [B, pages, Hkv, page, d]
    x = x.transpose(1, 2).flatten(2, 3)[:, :, :s["longest"]]
    return x if scale is None else x * scale[:, None, None]


def _plain_attn(s):
    c = s["case"]
    B, Lq, Hq, Hkv, d = c["B"], c["Lq"], c["Hq"], c["Hkv"], c["d"]
    g, lens = Hq // Hkv, s["lens"].long()
    asks = s["asks"].long() if c["ragged"] else torch.full_like(lens, Lq)
    keys, values = _gathered(s, s["cache_k"], s["ks"]), _gathered(s, s["cache_v"], s["vs"])
    q = s["q"].float().view(B, Lq, Hkv, g, d).permute(0, 2, 1, 3, 4).reshape(B, Hkv, Lq * g, d)
    score = torch.matmul(q, keys.transpose(2, 3)).view(B, Hkv, Lq, g, -1) / math.sqrt(d)
    at, row = torch.arange(s["longest"], device=DEV), torch.arange(Lq, device=DEV)
    seen = (at < lens[:, None])[:, None].expand(B, Lq, -1)
    if c["bs"]:
        pos = (lens - asks)[:, None] + row
        seen = seen & (at < (torch.div(pos, c["bs"], rounding_mode="floor") + 1)[:, :, None] * c["bs"])
    score = score.masked_fill(~seen[:, None, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), values).view(B, Hkv, Lq, g, d) / torch.where(total > 0, total, torch.ones_like(total))
    o = o.permute(0, 2, 1, 3, 4).reshape(B, Lq, Hq, d).to(BF16)
    lse = (top + total.log()).squeeze(-1).permute(0, 1, 3, 2).reshape(B, Hq, Lq)
    if c["ragged"]:
        live = row < asks[:, None]
        o, lse = torch.where(live[:, :, None, None], o, s["out"]), torch.where(live[:, None], lse, s["lse"])
    return dict(out=o, lse=lse)


_PLAIN = dict(qk_fwd=_plain_qk, qk_bwd=_plain_qk_bwd, append=_plain_append, attn=_plain_attn)


# ---- the library's calls --------------------------------------------------------------------------------------------
def _how(s):
    from paper_2604_04215_amd import binding as dlm
    return dict(q_weight=s["qw"], k_weight=s["kw"], eps=EPS, rope=s["rope"], positions=s["pos"], rope_style=dlm.ROPE_PAIRS if s["case"]["pairs"] else dlm.ROPE_HALVES)


def _workspace(s, nbytes):
    """Kept by the program from its first call on, as the other calls' workspaces are."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(16, nbytes()), dtype=U8, device=DEV)
    return s["ws"]


def _own_qk(s):
    from paper_2604_04215_amd import binding as dlm
    dlm.qk_norm_rope(s["q"], s["k"], s["q_out"], s["k_out"], **_how(s))
    return dict(q=s["q_out"], k=s["k_out"])


def _own_qk_bwd(s):
    from paper_2604_04215_amd import binding as dlm
    c, norm = s["case"], s["case"]["norm"]
    ws = _workspace(s, lambda: dlm.qk_norm_rope_bwd_workspace_bytes(c["T"], c["Hq"], c["Hkv"], c["d"]))
    given = dict(q=s["q"], k=s["k"], d_q_weight=s["dqw"], d_k_weight=s["dkw"], workspace=ws) if norm else {}
    dlm.qk_norm_rope_bwd(s["d_q_out"], s["d_k_out"], s["q_out"], s["k_out"], **given, **_how(s))
    got = dict(d_q=s["q_out"], d_k=s["k_out"])
    return dict(got, d_qw=s["dqw"], d_kw=s["dkw"]) if norm else got


def _own_append(s):
    from paper_2604_04215_amd import binding as dlm
    dlm.paged_append(s["k"], s["v"], s["cache_k"], s["cache_v"], s["slots"], q=s["q"], q_out=s["q_out"], k_scale=s["ks"], v_scale=s["vs"], **_how(s))
    return dict(q=s["q_out"], cache_k=s["cache_k"], cache_v=s["cache_v"])


def _own_attn(s):
    from paper_2604_04215_amd import binding as dlm
    c = s["case"]
    how = dict(max_kv_len=s["longest"], q_len=s["asks"], lse=s["lse"], k_scale=s["ks"], v_scale=s["vs"])
    if c["bs"]:
        how.update(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=c["bs"])
    given = (s["q"], s["out"], s["cache_k"], s["cache_v"], s["table"], s["lens"])
    ws = _workspace(s, lambda: dlm.paged_attn_workspace_bytes(*given, **how))
    dlm.paged_attn(*given, workspace=ws, **how)
    return dict(out=s["out"], lse=s["lse"])


_OWN = dict(qk_fwd=_own_qk, qk_bwd=_own_qk_bwd, append=_own_append, attn=_own_attn)


# --------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    with torch.enable_grad():
        return _EXACT[case["kind"]](prepare(case, seed))


def _define(s, x, w):
    """Norm and rotation of x [T, H, d] in 64 bits, the rotation as a product of complex numbers."""
    rot = s["case"]["rot"]
    if w is not None:
        x = x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt() * w
    if not rot:
        return x
    turn = torch.complex(*s["rope"].double()[s["pos"].long()].chunk(2, dim=1))[:, None]
    head = x[..., :rot].unflatten(-1, (rot // 2, 2) if s["case"]["pairs"] else (2, rot // 2))
    first, second = head.unbind(-1 if s["case"]["pairs"] else -2)
    z = torch.complex(first, second) * turn
    turned = torch.stack([z.real, z.imag], dim=-1 if s["case"]["pairs"] else -2).flatten(-2)
    return torch.cat([turned, x[..., rot:]], dim=-1)


def _wide(w):
    return None if w is None else w.double()


def _exact_qk(s):
    return dict(q=_define(s, s["q"].double(), _wide(s["qw"])), k=_define(s, s["k"].double(), _wide(s["kw"])))


def _exact_qk_bwd(s):
    got = {}
    for name in ("q", "k"):
        x, w = s[name].double().requires_grad_(), _wide(s[name + "w"])
        leaves = [x] if w is None else [x, w.requires_grad_()]
        grads = torch.autograd.grad(_define(s, x, w), leaves, s["d_" + name + "_out"].double())
        got["d_" + name] = grads[0]
        if w is not None:
            got["d_" + name + "w"] = grads[1]
    return got


def _exact_append(s):
    """The pages hold the quotients themselves where the calls hold the nearest of 8 or 16 bits."""
    c, page = s["case"], s["case"]["page"]
    q, k, v = _define(s, s["q"].double(), _wide(s["qw"])), _define(s, s["k"].double(), _wide(s["kw"])), s["v"].double()
    got = dict(q=q)
    live = torch.nonzero(s["slots"] >= 0).flatten()
    slots = s["slots"][live].long()
    for name, x, scale in (("cache_k", k, s["ks"]), ("cache_v", v, s["vs"])):
        if scale is not None:
            x = (x / scale.double()[None, :, None]).clamp(-LARGEST, LARGEST)
        rows = s[name].double().transpose(1, 2).reshape(-1, c["Hkv"], c["d"])
        rows[slots] = x[live]
        got[name] = rows.view(-1, page, c["Hkv"], c["d"]).transpose(1, 2).contiguous()
    return got


def _exact_attn(s):
    c = s["case"]
    Lq, Hq, Hkv, d = c["Lq"], c["Hq"], c["Hkv"], c["d"]
    out, lse = s["out"].double(), s["lse"].double()
    for b, n in enumerate(s["lens"].tolist()):
        asks = int(s["asks"][b]) if c["ragged"] else Lq
        held = s["table"][b, :-(-n // c["page"])].long()
        k, v = (_bits(x)[held].view(x.dtype).double().transpose(0, 1).reshape(Hkv, -1, d)[:, :n] for x in (s["cache_k"], s["cache_v"]))
        if c["e4m3"]:
            k, v = k * s["ks"].double()[:, None, None], v * s["vs"].double()[:, None, None]
        k, v = (x.repeat_interleave(Hq // Hkv, dim=0) for x in (k, v))
        logits = torch.einsum("ihd,hjd->hij", s["q"][b, :asks].double(), k) / math.sqrt(d)
        if c["bs"]:
            block_of = lambda p: torch.div(p, c["bs"], rounding_mode="floor")
            late = block_of(torch.arange(n, device=DEV))[None] > block_of(n - asks + torch.arange(asks, device=DEV))[:, None]
            logits = logits.masked_fill(late[None], -math.inf)
        z = torch.logsumexp(logits, dim=-1)
        p = torch.exp(logits - torch.where(z == -math.inf, torch.zeros_like(z), z)[..., None])
        out[b, :asks] = torch.einsum("hij,hjd->ihd", p, v)
        lse[b, :, :asks] = z
    return dict(out=out, lse=lse)


_EXACT = dict(qk_fwd=_exact_qk, qk_bwd=_exact_qk_bwd, append=_exact_append, attn=_exact_attn)


# --------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------------------------
def work(case):
    c, kind = case, case["kind"]
    Hq, Hkv, d = c["Hq"], c["Hkv"], c["d"]
    if kind in ("qk_fwd", "qk_bwd"):
        entries = float(c["T"]) * (Hq + Hkv) * d
        small = 4.0 * c["T"] + 4.0 * min(c["T"], c["seq"]) * c["rot"]          # positions, and each used row of the table once
        # forward: in and out; backward: the gradient in and out, and the heads again for the norm
        return dict(bytes=small + entries * (4.0 if kind == "qk_fwd" or not c["norm"] else 6.0), flops=entries * (8.0 if kind == "qk_fwd" else 16.0))
    if kind == "append":
        T, e = float(sum(_lengths(c, c["lo"], c["hi"]))), 1.0 if c["e4m3"] else 2.0
        entries = T * (Hq + 2 * Hkv) * d
        # (padding tokens' queries are rotated too)
        nbytes = 4.0 * (T + c["padded"]) * Hq * d + (2.0 + e) * 2 * T * Hkv * d + 8.0 * (T + c["padded"]) + 4.0 * min(T, c["before"] + c["hi"]) * c["rot"]
        return dict(bytes=nbytes, flops=entries * 8.0)
    lens = _lengths(c, c["lo"], c["hi"])
    asks = _lengths(c, 0, c["Lq"]) if c["ragged"] else [c["Lq"]] * c["B"]
    rows = float(sum(asks)) * Hq
    pairs = float(sum(n * a for n, a in zip(lens, asks))) * Hq
    keys = float(sum(n for n, a in zip(lens, asks) if a))
    return dict(bytes=2.0 * (1 if c["e4m3"] else 2) * keys * Hkv * d + rows * (4.0 * d + 4.0) + 4.0 * keys / c["page"], flops=4.0 * pairs * d)
