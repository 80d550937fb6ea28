"""The two ends of a training step with what lies between them: tokens -> embedding -> norm -> head norms and rotation -> attention -> residual and norm ->
log-likelihood of the masked tokens under the same table, and the gradients back to that table (GPU)."""
import numpy as np
import pytest
import torch

from oracle import heads
from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV

pytestmark = pytest.mark.gpu
BF16, F32, I32, U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
H = 2.0 ** -8                                            # half a step of bf16


def space(n):
    return torch.full((max(16, n),), 255, dtype=U8, device=DEV)


class Step:
    """Packed sequences (one of them empty, one of a single token) and three padding rows behind the last.  Dh = (Hq + 2 Hkv) d: the normed row is the heads, the
    attention's output is added to the first Hq d entries of the stream."""
    cu, T, Hq, Hkv, d, V, eps, scale = [0, 37, 37, 38, 101], 104, 4, 2, 64, 1003, 1e-5, 4.0
    Dh, forbid, temperature = 512, 1002, 0.8

    def __init__(self, table_type, layer):
        rng = np.random.default_rng(11)
        n = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32))
        self.layer, T, Dh = layer, self.T, self.Dh
        self.table = (n(self.V, Dh) * Dh ** -0.5 * 2).to(BF16).to(DEV)
        self.norm, self.bias = [(1 + 0.2 * n(Dh)).to(BF16).to(DEV) for _ in range(2)], [(0.2 * n(Dh)).to(BF16).to(DEV) if layer else None for _ in range(2)]
        self.heads = [(1 + 0.2 * n(self.d)).to(BF16).to(DEV) for _ in range(2)]
        self.rope = torch.from_numpy(heads.angles(64, self.d).astype(np.float32)).to(DEV)
        pos = np.concatenate([np.arange(b - a) for a, b in zip(self.cu, self.cu[1:])] + [np.zeros(3)])
        self.pos, self.dev_cu = torch.from_numpy(pos.astype(np.int32)).to(DEV), torch.tensor(self.cu, dtype=I32, device=DEV)
        self.tokens, self.target, self.mask = (torch.zeros(T, dtype=t, device=DEV) for t in (I32, I32, U8))
        self.weight = torch.zeros(T, device=DEV)
        b16 = lambda *s: torch.zeros(s, dtype=BF16, device=DEV)
        f32 = lambda *s: torch.zeros(s, dtype=F32, device=DEV)
        self.x, self.y, self.x2, self.y2, self.a, self.qkv = (b16(T, Dh) for _ in range(6))
        self.attn_lse, self.lse, self.zt, self.conf, self.tok, self.value = f32(self.Hq, T), f32(T), f32(T), f32(T), torch.zeros(T, dtype=I32, device=DEV), f32(1)
        self.rows, self.count, self.d_zt, self.d_lse = torch.zeros(T, dtype=I32, device=DEV), torch.zeros(1, dtype=I32, device=DEV), f32(T), f32(T)
        self.dy2, self.dx2, self.dqkv, self.dy, self.dx = (b16(T, Dh) for _ in range(5))
        self.d_table = torch.zeros((self.V, Dh), dtype=table_type, device=DEV)
        self.d_norm, self.d_bias, self.d_heads = [f32(Dh) for _ in range(2)], [f32(Dh) if layer else None for _ in range(2)], [f32(self.d) for _ in range(2)]
        self.how = dict(row_idx=self.rows, m_dev=self.count, target=self.target, forbid_token=self.forbid, inv_temperature=1 / self.temperature, out_scatter=True)
        self.back = dict(self.how, d_ztarget=self.d_zt, d_lse=self.d_lse, d_hidden=self.dy2, d_w=self.d_table, M=T)
        self.ws = [space(k) for k in (dlm.lmhead_workspace_bytes(T, self.V), dlm.lmhead_bwd_workspace_bytes(self.y2, self.table, self.lse, **self.back),
                                      dlm.row_norm_bwd_workspace_bytes(T, Dh), dlm.block_attn_bwd_workspace_bytes(T, self.Hq),
                                      dlm.qk_norm_rope_bwd_workspace_bytes(T, self.Hq, self.Hkv, self.d), dlm.embed_bwd_workspace_bytes(T, self.V, Dh))]

    def draw(self, seed, masked):
        rng = np.random.default_rng(seed)
        tokens, target = rng.integers(0, 40, self.T), rng.integers(0, self.forbid, self.T)       # (few different tokens: rows of the table that many add to)
        tokens[::7] = rng.integers(0, self.V, len(tokens[::7]))
        tokens[101:] = -1
        mask = rng.random(self.T) < masked
        mask[101:] = False
        weight = np.where(mask, rng.uniform(0.5, 2, self.T), 0.0)
        for t, v in ((self.tokens, tokens), (self.target, target), (self.mask, mask), (self.weight, weight)):
            t.copy_(torch.from_numpy(v))

    def split(self, t):
        return [u.unflatten(1, (-1, self.d)) for u in t.split([self.Hq * self.d, self.Hkv * self.d, self.Hkv * self.d], dim=1)]

    def forward(self):
        kind = dict(kind=dlm.NORM_LAYER if self.layer else dlm.NORM_RMS, eps=self.eps)
        dlm.embed(self.tokens, self.table, self.x, scale=self.scale)
        dlm.row_norm(self.x, self.y, weight=self.norm[0], bias=self.bias[0], **kind)
        (q0, k0, v), (q, k, _), wide = self.split(self.y), self.split(self.qkv), self.Hq * self.d
        dlm.qk_norm_rope(q0, k0, q, k, q_weight=self.heads[0], k_weight=self.heads[1], rope=self.rope, positions=self.pos)
        self.split(self.qkv)[2].copy_(v)
        q, k, v = self.split(self.qkv)
        dlm.varlen_attn(q, k, v, self.a[:, :wide].unflatten(1, (-1, self.d)), self.dev_cu, 64, lse=self.attn_lse)
        dlm.row_norm(self.a, self.y2, residual=self.x, sum_out=self.x2, weight=self.norm[1], bias=self.bias[1], **kind)
        dlm.mask_compact(self.mask[None], self.rows, self.count)
        dlm.lmhead_confidence(self.y2, self.table, self.conf, self.tok, lse=self.lse, ztarget=self.zt, workspace=self.ws[0], M=self.T, **self.how)
        self.d_zt.copy_(self.weight)
        self.d_lse.copy_(-self.weight)
        dlm.seq_logprob(self.zt[None], self.lse[None], self.mask[None], self.value)

    def backward(self):
        kind, wide = dict(kind=dlm.NORM_LAYER if self.layer else dlm.NORM_RMS, eps=self.eps), self.Hq * self.d
        self.dy2.zero_()                                 # (rows that are not masked are not written)
        dlm.lmhead_bwd(self.y2, self.table, self.lse, workspace=self.ws[1], **self.back)
        dlm.row_norm_bwd(self.dy2, self.x2, self.dx2, weight=self.norm[1], d_weight=self.d_norm[1], d_bias=self.d_bias[1], workspace=self.ws[2], **kind)
        (q, k, v), (dq, dk, dv) = self.split(self.qkv), self.split(self.dqkv)
        heads_of = lambda t: t[:, :wide].unflatten(1, (-1, self.d))
        dlm.block_attn_bwd(q, heads_of(self.a), heads_of(self.dx2), self.attn_lse, dq, block=(k, v), d_block=(dk, dv), cu_seqlens=self.dev_cu, max_seqlen=64,
                           workspace=self.ws[3])
        (q0, k0, _), (eq, ek, ev) = self.split(self.y), self.split(self.dy)
        dlm.qk_norm_rope_bwd(dq, dk, eq, ek, q=q0, k=k0, q_weight=self.heads[0], k_weight=self.heads[1], d_q_weight=self.d_heads[0], d_k_weight=self.d_heads[1],
                             rope=self.rope, positions=self.pos, workspace=self.ws[4])
        ev.copy_(dv)
        dlm.row_norm_bwd(self.dy, self.x, self.dx, weight=self.norm[0], d_sum=self.dx2, d_weight=self.d_norm[0], d_bias=self.d_bias[0], workspace=self.ws[2], **kind)
        dlm.embed_bwd(self.tokens, self.dx, self.d_table, scale=self.scale, accumulate=True, workspace=self.ws[5])

    def results(self):
        return [self.value, self.d_table, *self.d_norm, *self.d_heads] + ([*self.d_bias] if self.layer else [])

    def value64(self, table, norm, head, bias):
        """(the masked tokens' weighted log-likelihood, the same without weights), in 64 bits on the CPU"""
        tokens, mask, target, weight = self.tokens.cpu().long(), self.mask.cpu().bool(), self.target.cpu().long(), self.weight.cpu().double()
        rope, pos = self.rope.cpu().double(), self.pos.cpu().long()

        def normed(x, w, b):
            if self.layer:
                x = x - x.mean(-1, keepdim=True)
            y = x / (x.square().mean(-1, keepdim=True) + self.eps).sqrt() * w
            return y if b is None else y + b

        def rotated(x, w):
            x = x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt() * w
            c, s = (t[:, None] for t in rope[pos].chunk(2, 1))
            a, b = x.chunk(2, -1)
            return torch.cat([a * c - b * s, b * c + a * s], -1)

        x = self.scale * table[tokens.clamp(min=0)] * (tokens >= 0)[:, None]
        q, k, v = self.split(normed(x, norm[0], bias[0]))
        q, k, out = rotated(q, head[0]), rotated(k, head[1]), torch.zeros_like(x)
        for a, b in zip(self.cu, self.cu[1:]):
            if a < b:
                g = self.Hq // self.Hkv
                s = torch.einsum("ihd,jhd->hij", q[a:b], k[a:b].repeat_interleave(g, 1)) / self.d ** 0.5
                out[a:b, :self.Hq * self.d] = torch.einsum("hij,jhd->ihd", s.softmax(-1), v[a:b].repeat_interleave(g, 1)).flatten(1)
        z = normed(x + out, norm[1], bias[1]) @ table.T / self.temperature
        z = torch.cat([z[:, :self.forbid], torch.full_like(z[:, :1], -torch.inf)], 1)
        logp = z.log_softmax(-1).gather(1, target[:, None])[:, 0][mask]
        return (weight[mask] * logp).sum(), logp.sum()


@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("table_type", [BF16, F32])
@pytest.mark.parametrize("masked", [0.4, 1.0, 0.0])
def test_gradients_of_a_step(masked, table_type, layer):
    """Against 64-bit automatic differentiation.  A result lies behind at most 16 roundings of whole tensors to bf16 (forward 8: stream, norm, heads, probabilities, output,
    sum, norm, value; backward 8: dz, two norms, three of attention, heads, table), each of 2^-8 / sqrt(3) of the tensor in the norm and carried on with
    factors near one (normed rows, logits of size 2).  Should all add up: 16 * 2.3e-3 = 3.6e-2."""
    s = Step(table_type, layer)
    s.draw(5, masked)
    s.d_table.fill_(float("nan"))                        # written by the LM head's gradient, then added to
    s.forward()
    s.backward()
    torch.cuda.synchronize()
    leaves = [t.detach().double().cpu().requires_grad_() for t in (s.table, *s.norm, *s.heads, *(s.bias if layer else []))]
    total, plain = s.value64(leaves[0], leaves[1:3], leaves[3:5], leaves[5:] if layer else [None] * 2)
    plain = float(plain.detach())
    assert abs(float(s.value) - plain) <= 3.6e-2 * max(1.0, abs(plain))
    if masked == 0:
        assert all((t == 0).all() for t in s.results())
        return
    for got, want in zip(s.results()[1:], torch.autograd.grad(total, leaves)):
        rel = float((got.double().cpu() - want).norm() / want.norm())
        assert rel <= 16 * H / 3 ** 0.5, (tuple(want.shape), rel)


@pytest.mark.parametrize("table_type", [BF16, F32])
def test_a_step_replayed_from_a_graph(table_type):
    """Other tokens and other masks (none, all) between the replays, the program's own eager steps and another stream beside them."""
    eager, caught, aside = (Step(table_type, False) for _ in range(3))
    caught.draw(1, 0.5)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    caught.forward()
    caught.backward()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        caught.forward()
        caught.backward()
    for seed, masked in ((1, 0.5), (2, 0.0), (3, 1.0), (4, 0.1), (1, 0.5)):
        for s in (eager, caught, aside):
            s.draw(seed, masked)
            for t in s.ws:
                t.fill_(255)
            s.d_table.fill_(7.0)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            aside.forward()
            aside.backward()
        graph.replay()
        eager.forward()
        eager.backward()
        torch.cuda.synchronize()
        for other in (caught, aside):
            assert all(torch.equal(a, b) for a, b in zip(eager.results(), other.results())), (seed, masked)
