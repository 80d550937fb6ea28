"""The two ends of a training step, as timed cases: what they compute in plain torch, and the library's calls.

Five kinds, each one entry point of `binding`:

  embed      rows of the embedding table for a batch of tokens, scaled
  embed_bwd  their gradient: rows of equal tokens summed (half of a masked batch is one token, <MASK>)
  norm       RMS or layer norm of the rows between two layers, with the residual added on the way in
  norm_bwd   its gradient: rows, with the residual stream's own gradient added, weight and bias
  lmhead_bwd gradient of the LM head's log-sum-exp and target logit: hidden rows and vocabulary weights, no logits kept

`own` says which of the two `run` takes.  Sizes are those of the workloads in `synth`, of the tests and of the benchmark (vocabularies of 300 to
157184, hidden sizes of 64 to 4096, blocks of 32, groups of 8, packed batches of 64 k tokens) and sizes around them; hidden rows and gradients are
N(0, 1), the vocabulary's weights N(0, Dh^(-1/2)) as there.
"""
import math
import random

import torch

own = False

BF16, F32, F64, I32, I64, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64, torch.uint8
DEV = "cuda:0"


# --------------------------------------------------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------------------------------------------------
def _embed(T, V, Dh, masked, padded, f32, scale):
    """T tokens, a share `masked` of them <MASK> (the last id), the last `padded` none at all; f32: rows of 32 bits come out."""
    return dict(kind="embed", T=T, V=V, Dh=Dh, masked=masked, padded=padded, f32=f32, scale=scale)


def _embed_bwd(T, V, Dh, masked, padded, f32, scale, rows32, accumulate):
    """Gradient of the above; rows32: upstream rows of 32 bits; f32: a table of 32 bits; accumulate: added to what the table holds."""
    return dict(_embed(T, V, Dh, masked, padded, f32, scale), kind="embed_bwd", rows32=rows32, accumulate=accumulate)


def _norm(kind, T, D, layer, affine, f32, residual):
    """T rows of D entries; affine: 0 no weight, 1 weight, 2 weight and bias; f32: rows (and residual) of 32 bits; residual: a second input is added
    and the sum comes out too (backward: the sum's own gradient is added)."""
    return dict(kind=kind, T=T, D=D, layer=layer, affine=affine, f32=f32, residual=residual)


def _head(M, rows, Dh, V, f32, forbid, temperature, zloss, accumulate=False):
    """M masked rows of `rows` hidden ones; f32: gradients of 32 bits; forbid: the last id cannot be predicted; zloss: weight of a second term,
    lse squared; accumulate: the weights' gradient is added to what its buffer holds."""
    return dict(kind="lmhead_bwd", M=M, rows=rows, Dh=Dh, V=V, f32=f32, forbid=forbid, temperature=temperature, zloss=zloss, accumulate=accumulate)


def listed():
    return [
        # one denoising step of the benchmark's default rollout (8 sequences, blocks of 32): latency
        dict(_embed(256, 126464, 4096, 0.5, 0, False, 1.0), name="embed_block"),
        # the packed batch of an actor update, 64 k tokens, into a residual stream of 32 bits, scaled by the root of the hidden size
        dict(_embed(65536, 126464, 4096, 0.5, 77, True, 64.0), name="embed_packed"),
        # a micro-batch of a small model, a whole gradient in 32 bits
        dict(_embed_bwd(333, 2048, 256, 0.4, 5, True, 1.0, False, False), name="embed_bwd_small"),
        # 8 sequences of 1024 tokens, the whole 16-bit gradient of a large table: mostly rows of zeros
        dict(_embed_bwd(8192, 152064, 3584, 0.5, 0, False, 1.0, False, False), name="embed_bwd_dense"),
        # the packed batch, added to a gradient that is kept in 32 bits over micro-batches (or shared with the LM head)
        dict(_embed_bwd(65536, 126464, 4096, 0.5, 77, True, 64.0, False, True), name="embed_bwd_packed"),
        # between two layers of a denoising step: residual added, RMS norm
        dict(_norm("norm", 256, 4096, False, 1, False, True), name="norm_block"),
        # training forward over the packed batch, layer norm with a bias, rows of 32 bits
        dict(_norm("norm", 65536, 3584, True, 2, True, False), name="norm_layer_packed"),
        # a micro-batch of a small model (14 heads of 64), layer norm
        dict(_norm("norm_bwd", 333, 896, True, 2, False, False), name="norm_bwd_small"),
        # the actor update's packed batch, RMS norm inside a residual stream
        dict(_norm("norm_bwd", 65536, 4096, False, 1, False, True), name="norm_bwd_packed"),
        # the loss of one half-masked block of a small model, gradients in 32 bits
        dict(_head(16, 32, 256, 2048, True, True, 1.0, 0.0), name="lmhead_bwd_small"),
        # the masked positions of 16 blocks of 32: reading and writing the vocabulary's weights takes as long as the products
        dict(_head(512, 512, 4096, 126464, False, True, 1.0, 0.0), name="lmhead_bwd_blocks"),
        # a training micro-batch, half of 8192 positions masked
        dict(_head(4096, 8192, 3584, 152064, False, True, 1.0, 0.0), name="lmhead_bwd_batch"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


_WIDTHS = [64, 192, 256, 320, 896, 1024, 1536, 2048, 2560, 3584, 4096]


def draw(rng):
    kind = rng.choice(["embed", "embed_bwd", "embed_bwd", "norm", "norm_bwd", "lmhead_bwd", "lmhead_bwd"])
    D, f32 = rng.choice(_WIDTHS), rng.random() < 0.4
    if kind in ("norm", "norm_bwd"):
        T = _log(rng, 1, min(131072, 65536 * 3584 // D))
        return _norm(kind, T, rng.choice([D, D, 8 * _log(rng, 1, D // 8)]), rng.random() < 0.5, rng.choice([0, 1, 1, 2, 2]), f32 and (kind == "norm" or T * D < 1 << 27), rng.random() < 0.5)
    V = _log(rng, 300, 157184)
    if kind == "lmhead_bwd":
        M = _log(rng, 1, min(8192, 4096 * 3584 * 152064 // (D * V)))
        f32 = f32 and 16 <= M and M * V * D < 1 << 39
        return _head(M, M + rng.choice([0, _log(rng, 1, 1 + M)]), D, V, f32, rng.random() < 0.7, rng.choice([1.0, 1.0, 0.7]), rng.choice([0.0, 0.0, 1e-3]), rng.random() < 0.3)
    T = _log(rng, 1, min(131072, 65536 * 4096 // D))
    masked, padded, scale = rng.choice([0.0, 0.15, 0.5, 0.9, 1.0]), rng.choice([0, 0, min(T, _log(rng, 1, 100))]), rng.choice([1.0, 1.0, math.sqrt(D)])
    if kind == "embed":
        return _embed(T, V, D, masked, padded, f32, scale)
    return _embed_bwd(T, V, D, masked, padded, f32, scale, rng.random() < 0.3 and T * D < 1 << 27, rng.random() < 0.5)


# --------------------------------------------------------------------------------------------------------------------
# what a user has in hand before the call
# --------------------------------------------------------------------------------------------------------------------
class _Draw:
    """Seeded draws on the GPU; ids on the host, which is quick enough for them."""

    def __init__(self, seed):
        self.g = torch.Generator(device=DEV).manual_seed(seed)
        self.host = torch.Generator().manual_seed(seed)

    def normal(self, *shape, dtype=BF16):
        return torch.randn(shape, generator=self.g, device=DEV, dtype=dtype)

    def vocabulary(self, V, Dh):
        return self.normal(V, Dh).mul_(Dh ** -0.25)

    def around(self, mean, n):
        return (mean + 0.2 * torch.randn(n, generator=self.g, device=DEV)).to(BF16)

    def ids(self, n, V):
        """Ids as text has them: few frequent ones, a long tail."""
        return torch.exp(torch.rand(n, generator=self.host, dtype=F64) * math.log(V)).floor().to(I64).clamp_(1, V) - 1


def _tokens(c, r):
    x = r.ids(c["T"], c["V"])
    x[torch.rand(c["T"], generator=r.host) < c["masked"]] = c["V"] - 1
    if c["padded"]:
        x[-c["padded"]:] = -1
    return x.to(I32)


def prepare(case, seed):
    return _PREPARE[case["kind"]](case, _Draw(seed))


def _prepare_embed(c, r):
    s = dict(kind=c["kind"], case=c, tokens=_tokens(c, r).to(DEV))
    if c["kind"] == "embed":
        s["table"] = r.vocabulary(c["V"], c["Dh"])
        s["out"] = torch.zeros((c["T"], c["Dh"]), dtype=F32 if c["f32"] else BF16, device=DEV)
        return s
    s["d_out"] = r.normal(c["T"], c["Dh"], dtype=F32 if c["rows32"] else BF16)
    kept = F32 if c["f32"] else BF16
    s["d_table"] = r.normal(c["V"], c["Dh"], dtype=kept) if c["accumulate"] else torch.zeros((c["V"], c["Dh"]), dtype=kept, device=DEV)
    return s


def _prepare_norm(c, r):
    T, D, t = c["T"], c["D"], F32 if c["f32"] else BF16
    s = dict(kind=c["kind"], case=c, x=r.normal(T, D, dtype=t), eps=1e-5 if c["layer"] else 1e-6)
    if c["layer"]:
        s["x"].add_(r.normal(T, 1, dtype=t))            # rows of different means
    s["weight"] = r.around(1.0, D) if c["affine"] else None
    s["bias"] = r.around(0.0, D) if c["affine"] == 2 else None
    extra = r.normal(T, D, dtype=t) if c["residual"] else None
    if c["kind"] == "norm":
        s["residual"], s["sum"] = extra, torch.zeros_like(s["x"]) if c["residual"] else None
        s["out"] = torch.zeros((T, D), dtype=BF16, device=DEV)
        return s
    s["d_sum"], s["d_out"], s["d_x"] = extra, r.normal(T, D), torch.zeros_like(s["x"])
    s["d_weight"] = torch.zeros(D, dtype=F32, device=DEV) if c["affine"] else None
    s["d_bias"] = torch.zeros(D, dtype=F32, device=DEV) if c["affine"] == 2 else None
    return s


def _prepare_head(c, r):
    """Rows whose target gets between none and most of the probability, as over the course of a training."""
    M, rows, Dh, V = c["M"], c["rows"], c["Dh"], c["V"]
    forbid = V - 1 if c["forbid"] else -1
    s = dict(kind="lmhead_bwd", case=c, w=r.vocabulary(V, Dh), forbid=forbid)
    chosen = torch.randperm(rows, generator=r.host)[:M].sort().values.to(DEV)
    target = r.ids(M, V - 1).to(DEV)
    hidden = r.normal(rows, Dh, dtype=F32)
    pull = s["w"][target].float()
    largest = math.sqrt(2.0 * math.log(V)) * Dh ** 0.25          # of the other logits, about
    wanted = largest * torch.rand((M, 1), generator=r.g, device=DEV)
    hidden[chosen] += pull / pull.square().sum(1, keepdim=True) * (wanted - (hidden[chosen] * pull).sum(1, keepdim=True))
    s["hidden"] = hidden.to(BF16)
    z = torch.matmul(s["hidden"][chosen].float(), s["w"].float().t()) / c["temperature"]
    if c["forbid"]:
        z[:, forbid] = -math.inf
    lse = torch.logsumexp(z, 1)
    # the terms of the log-likelihood, weighted by 1 / t of their sequence, and the squared lse's
    g = -(1.0 + 9.0 * torch.rand(M, generator=r.g, device=DEV)) / rows
    for name, x in (("lse", lse), ("d_ztarget", g), ("d_lse", -g + 2.0 * c["zloss"] / rows * lse)):
        s[name] = torch.zeros(rows, dtype=F32, device=DEV)
        s[name][chosen] = x
    s["target"] = torch.zeros(rows, dtype=I32, device=DEV)
    s["target"][chosen] = target.to(I32)
    s["chosen"] = chosen.to(I32)
    kept = F32 if c["f32"] else BF16
    s["d_hidden"] = torch.zeros((rows, Dh), dtype=kept, device=DEV)
    s["d_w"] = r.normal(V, Dh, dtype=kept).mul_(1e-3) if c["accumulate"] else torch.zeros((V, Dh), dtype=kept, device=DEV)
    return s


_PREPARE = dict(embed=_prepare_embed, embed_bwd=_prepare_embed, norm=_prepare_norm, norm_bwd=_prepare_norm, lmhead_bwd=_prepare_head)


# --------------------------------------------------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------------------------------------------------
def run(state):
    return (_OWN if own else _PLAIN)[state["kind"]](state)


# ---- in plain torch -------------------------------------------------------------------------------------------------
def _plain_embed(s):
    live = s["tokens"] >= 0
    rows = s["table"][s["tokens"].clamp(min=0).long()].float() * s["case"]["scale"]
    return dict(out=torch.where(live[:, None], rows, torch.zeros_like(rows)).to(s["out"].dtype))


def _plain_embed_bwd(s):
    """Rows in the order of their tokens; the sum of a token's is the difference of two running sums, in 64 bits."""
    c = s["case"]
    token, order = torch.where(s["tokens"] >= 0, s["tokens"], torch.full_like(s["tokens"], c["V"])).sort()
    running = torch.zeros((c["T"] + 1, c["Dh"]), dtype=F64, device=DEV)
    torch.cumsum(s["d_out"][order].double(), 0, out=running[1:])
    ids = torch.arange(c["V"], device=DEV, dtype=I32)
    total = (running[torch.searchsorted(token, ids, right=True)] - running[torch.searchsorted(token, ids)]) * c["scale"]
    if c["accumulate"]:
        total += s["d_table"]
    s["d_table"].copy_(total)
    return dict(d_table=s["d_table"])


def _normed(s, x):
    """x in 32 bits without mean (layer norm) and of unit size, and the factor that made it so."""
    if s["case"]["layer"]:
        x = x - x.mean(-1, keepdim=True)
    r = torch.rsqrt(x.square().mean(-1, keepdim=True) + s["eps"])
    return x * r, r


def _plain_norm(s):
    x = s["x"]
    if s["residual"] is not None:
        x = (x.float() + s["residual"].float()).to(x.dtype)
    y, _ = _normed(s, x.float())
    if s["weight"] is not None:
        y = y * s["weight"].float()
    if s["bias"] is not None:
        y = y + s["bias"].float()
    got = dict(out=y.to(BF16))
    return got if s["residual"] is None else dict(got, sum=x)


def _plain_norm_bwd(s):
    n, r = _normed(s, s["x"].float())
    dy = s["d_out"].float()
    g = dy if s["weight"] is None else dy * s["weight"].float()
    dx = g - n * (g * n).mean(-1, keepdim=True)
    if s["case"]["layer"]:
        dx = dx - g.mean(-1, keepdim=True)
    dx = dx * r
    if s["d_sum"] is not None:
        dx = dx + s["d_sum"].float()
    got = dict(d_x=dx.to(s["x"].dtype))
    if s["weight"] is not None:
        got["d_weight"] = (dy * n).double().sum(0).float()
    if s["bias"] is not None:
        got["d_bias"] = dy.double().sum(0).float()
    return got


def _plain_head(s):
    """Gradients of 32 bits take their exponents from logits of 64: an error of a logit is one of the probability."""
    c, at = s["case"], s["chosen"].long()
    M, wide = c["M"], F64 if c["f32"] else F32
    h, w = s["hidden"][at], s["w"]
    z = torch.matmul(h.to(wide), w.to(wide).t()) / c["temperature"]
    if c["forbid"]:
        z[:, s["forbid"]] = -math.inf
    dz = torch.exp(z - s["lse"][at][:, None]).float() * s["d_lse"][at][:, None]
    dz[torch.arange(M, device=DEV), s["target"][at].long()] += s["d_ztarget"][at]
    dz /= c["temperature"]
    s["d_hidden"][at] = torch.matmul(dz, w.float()).to(s["d_hidden"].dtype)
    d_w = torch.matmul(dz.t(), h.float())
    if c["accumulate"]:
        d_w += s["d_w"]
    s["d_w"].copy_(d_w)
    return dict(d_hidden=s["d_hidden"], d_w=s["d_w"])


_PLAIN = dict(embed=_plain_embed, embed_bwd=_plain_embed_bwd, norm=_plain_norm, norm_bwd=_plain_norm_bwd, lmhead_bwd=_plain_head)


# ---- the library's calls --------------------------------------------------------------------------------------------
def _workspace(s, nbytes):
    """Kept by the program from its first call on, as the other calls' workspaces are."""
    if "ws" not in s:
        s["ws"] = torch.empty(max(16, nbytes()), dtype=U8, device=DEV)
    return s["ws"]


def _own_embed(s):
    from paper_2604_04215_amd import binding as dlm
    dlm.embed(s["tokens"], s["table"], s["out"], scale=s["case"]["scale"])
    return dict(out=s["out"])


def _own_embed_bwd(s):
    from paper_2604_04215_amd import binding as dlm
    c = s["case"]
    ws = _workspace(s, lambda: dlm.embed_bwd_workspace_bytes(c["T"], c["V"], c["Dh"]))
    dlm.embed_bwd(s["tokens"], s["d_out"], s["d_table"], scale=c["scale"], accumulate=c["accumulate"], workspace=ws)
    return dict(d_table=s["d_table"])


def _own_norm(s):
    from paper_2604_04215_amd import binding as dlm
    dlm.row_norm(s["x"], s["out"], kind=dlm.NORM_LAYER if s["case"]["layer"] else dlm.NORM_RMS, weight=s["weight"], bias=s["bias"], eps=s["eps"],
                 residual=s["residual"], sum_out=s["sum"])
    return dict(out=s["out"]) if s["sum"] is None else dict(out=s["out"], sum=s["sum"])


def _own_norm_bwd(s):
    from paper_2604_04215_amd import binding as dlm
    c = s["case"]
    ws = _workspace(s, lambda: dlm.row_norm_bwd_workspace_bytes(c["T"], c["D"])) if c["affine"] else None
    dlm.row_norm_bwd(s["d_out"], s["x"], s["d_x"], kind=dlm.NORM_LAYER if c["layer"] else dlm.NORM_RMS, weight=s["weight"], eps=s["eps"], d_sum=s["d_sum"],
                     d_weight=s["d_weight"], d_bias=s["d_bias"], workspace=ws)
    return {k: s[k] for k in ("d_x", "d_weight", "d_bias") if s[k] is not None}


def _own_head(s):
    from paper_2604_04215_amd import binding as dlm
    c = s["case"]
    given = (s["hidden"], s["w"], s["lse"])
    how = dict(target=s["target"], d_ztarget=s["d_ztarget"], d_lse=s["d_lse"], d_hidden=s["d_hidden"], d_w=s["d_w"], accumulate=c["accumulate"], row_idx=s["chosen"],
               inv_temperature=1.0 / c["temperature"], forbid_token=s["forbid"], out_scatter=True)
    ws = _workspace(s, lambda: dlm.lmhead_bwd_workspace_bytes(*given, **how))
    dlm.lmhead_bwd(*given, workspace=ws, **how)
    return dict(d_hidden=s["d_hidden"], d_w=s["d_w"])


_OWN = dict(embed=_own_embed, embed_bwd=_own_embed_bwd, norm=_own_norm, norm_bwd=_own_norm_bwd, lmhead_bwd=_own_head)


# --------------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    with torch.enable_grad():
        return _EXACT[case["kind"]](prepare(case, seed))


def _exact_embed(s):
    out = torch.zeros(s["out"].shape, dtype=F64, device=DEV)
    live = torch.nonzero(s["tokens"] >= 0).flatten()
    out[live] = s["table"].index_select(0, s["tokens"][live]).double() * s["case"]["scale"]
    return dict(out=out)


def _exact_embed_bwd(s):
    """Every row added to its token's."""
    c = s["case"]
    got = s["d_table"].double() if c["accumulate"] else torch.zeros(s["d_table"].shape, dtype=F64, device=DEV)
    live = torch.nonzero(s["tokens"] >= 0).flatten()
    return dict(d_table=got.index_add_(0, s["tokens"][live], s["d_out"][live].double(), alpha=c["scale"]))


def _define_norm(s, x, w, b):
    """The definition in 64 bits: deviation from the mean (or from zero) over its root mean square."""
    d = x - x.sum(-1, keepdim=True) / x.shape[-1] if s["case"]["layer"] else x
    y = d / (d.pow(2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]).sqrt()
    y = y if w is None else y * w
    return y if b is None else y + b


def _wide(x):
    return None if x is None else x.double()


def _exact_norm(s):
    if s["residual"] is None:
        return dict(out=_define_norm(s, s["x"].double(), _wide(s["weight"]), _wide(s["bias"])))
    total = s["x"].double() + s["residual"].double()
    # what is normalised is the sum as it is kept
    return dict(out=_define_norm(s, total.to(s["x"].dtype).double(), _wide(s["weight"]), _wide(s["bias"])), sum=total)


def _exact_norm_bwd(s):
    x, w, b = s["x"].double().requires_grad_(), _wide(s["weight"]), _wide(s["bias"])
    leaves = dict(d_x=x)
    if w is not None:
        leaves["d_weight"] = w.requires_grad_()
    if b is not None:
        leaves["d_bias"] = b.requires_grad_()
    got = dict(zip(leaves, torch.autograd.grad(_define_norm(s, x, w, b), list(leaves.values()), s["d_out"].double())))
    if s["d_sum"] is not None:
        got["d_x"] = got["d_x"] + s["d_sum"].double()
    return got


def _exact_head(s):
    """Vocabulary slices, the one-hot of the target as a comparison."""
    c, at = s["case"], s["chosen"].long()
    h, lse, target = s["hidden"][at].double(), s["lse"][at].double(), s["target"][at]
    d_hidden, d_w = torch.zeros_like(s["hidden"], dtype=F64), s["d_w"].double() if c["accumulate"] else torch.zeros(s["d_w"].shape, dtype=F64, device=DEV)
    rows = torch.zeros_like(h)
    for v0 in range(0, c["V"], 16384):
        w = s["w"][v0:v0 + 16384].double()
        ids = torch.arange(v0, v0 + w.shape[0], device=DEV)
        p = torch.exp(h @ w.t() / c["temperature"] - lse[:, None]) * (ids != s["forbid"])
        dz = (s["d_lse"][at].double()[:, None] * p + s["d_ztarget"][at].double()[:, None] * (ids == target[:, None])) / c["temperature"]
        rows += dz @ w
        d_w[v0:v0 + w.shape[0]] += dz.t() @ h
    d_hidden[at] = rows
    return dict(d_hidden=d_hidden, d_w=d_w)


_EXACT = dict(embed=_exact_embed, embed_bwd=_exact_embed_bwd, norm=_exact_norm, norm_bwd=_exact_norm_bwd, lmhead_bwd=_exact_head)


# --------------------------------------------------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------------------------------------------------
class _Host(_Draw):
    """Ids alone, for the number of different ones."""

    def __init__(self):
        self.host = torch.Generator().manual_seed(1)


def work(case):
    c, kind = case, case["kind"]
    if kind in ("embed", "embed_bwd"):
        T, V, Dh, e = float(c["T"]), float(c["V"]), float(c["Dh"]), 4.0 if c["f32"] else 2.0
        ids = _tokens(c, _Host())
        distinct = float(ids[ids >= 0].unique().numel())
        if kind == "embed":
            return dict(bytes=4.0 * T + 2.0 * distinct * Dh + e * T * Dh, flops=T * Dh)
        live = T - c["padded"]
        return dict(bytes=4.0 * T + (4.0 if c["rows32"] else 2.0) * live * Dh + (2.0 * e * distinct if c["accumulate"] else e * V) * Dh, flops=live * Dh)
    if kind in ("norm", "norm_bwd"):
        entries, e = float(c["T"]) * c["D"], 4.0 if c["f32"] else 2.0
        if kind == "norm":
            return dict(bytes=entries * (2.0 + e * (3 if c["residual"] else 1)), flops=entries * 6.0)
        return dict(bytes=entries * (2.0 + e * (3 if c["residual"] else 2)), flops=entries * 12.0)
    M, Dh, V, e = float(c["M"]), float(c["Dh"]), float(c["V"]), 4.0 if c["f32"] else 2.0
    return dict(bytes=V * Dh * (2.0 + e * (2 if c["accumulate"] else 1)) + M * Dh * (2.0 + e) + 20.0 * M, flops=6.0 * M * V * Dh)
