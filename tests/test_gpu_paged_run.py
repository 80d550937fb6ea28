"""The paged operators together, as a block-diffusion engine runs them: prompts into the pages, then denoising steps of one block, each of
which stores the block's keys and values again, attends to everything in the pages and commits tokens; and the training side, forward and backward
through norm, rotation and attention (GPU)."""
import numpy as np
import pytest
import torch

from oracle import heads
from paper_2604_04215_amd import binding as dlm
from gpu_util import DEV
from test_gpu_paged_attn import U, H, compare, wide

pytestmark = pytest.mark.gpu
BF16, I32, E4M3 = torch.bfloat16, torch.int32, torch.float8_e4m3fn


class Engine:
    """Three sequences, pages of 16, blocks of 4."""
    page, Lb, Hq, Hkv, d, V, Dh = 16, 4, 4, 2, 64, 300, 64

    def __init__(self, e4m3, seed=3):
        self.rng = np.random.default_rng(seed)
        self.prompt = [37, 5, 64]
        B, total = 3, [n + self.Lb for n in self.prompt]
        counts = [-(-n // self.page) for n in total]
        order = self.rng.permutation(sum(counts) + 2)
        self.table = np.full((B, max(counts)), -1, dtype=np.int32)
        at = 0
        for b, m in enumerate(counts):
            self.table[b, :m] = order[at:at + m]
            at += m
        kind = E4M3 if e4m3 else BF16
        self.pages = [torch.zeros((len(order), self.Hkv, self.page, self.d), device=DEV).to(kind) for _ in range(2)]
        self.scales = [torch.tensor([0.05, 0.06], device=DEV) if e4m3 else None for _ in range(2)]
        self.w = [self.normal(self.d).abs().add(0.5).to(BF16) for _ in range(2)]
        self.rope = torch.from_numpy(heads.angles(128, self.d).astype(np.float32)).to(DEV)
        self.w_vocab = self.normal(self.V, self.Dh)
        self.x = torch.zeros((B, 128), dtype=I32, device=DEV)
        self.dev_table, self.kv_len = torch.from_numpy(self.table).to(DEV), torch.tensor(total, dtype=I32, device=DEV)

    def normal(self, *shape):
        return torch.from_numpy(self.rng.standard_normal(shape).astype(np.float32)).to(BF16).to(DEV)

    def append(self, qkv, seqs, pos):
        """Heads [T, Hq + 2 Hkv, d] of tokens at `pos` of sequences `seqs`; their queries come back."""
        slots = self.table[seqs, pos // self.page] * self.page + pos % self.page
        q, k, v = qkv.split([self.Hq, self.Hkv, self.Hkv], dim=1)
        out = torch.empty((len(pos), self.Hq, self.d), dtype=BF16, device=DEV)
        dlm.paged_append(k, v, *self.pages, torch.from_numpy(slots.astype(np.int32)).to(DEV), q=q, q_out=out, q_weight=self.w[0], k_weight=self.w[1],
                         rope=self.rope, positions=torch.from_numpy(pos.astype(np.int32)).to(DEV), k_scale=self.scales[0], v_scale=self.scales[1])
        return out


@pytest.mark.parametrize("e4m3", [False, True])
def test_prompts_then_steps_of_a_block(e4m3):
    g = Engine(e4m3)
    B, Lb = 3, g.Lb
    seqs = np.repeat(np.arange(B), g.prompt)
    pos = np.concatenate([np.arange(n) for n in g.prompt])
    prompt = g.normal(len(pos), g.Hq + 2 * g.Hkv, g.d)
    g.append(prompt, seqs, pos)
    block_seq, block_pos = np.repeat(np.arange(B), Lb), np.concatenate([n + np.arange(Lb) for n in g.prompt])
    mask = torch.ones((B, Lb), dtype=torch.uint8, device=DEV)
    conf, tok = torch.zeros((B, Lb), device=DEV), torch.zeros((B, Lb), dtype=I32, device=DEV)
    n_commit, remaining = (torch.zeros(B, dtype=I32, device=DEV) for _ in range(2))
    ws = torch.empty(dlm.lmhead_workspace_bytes(B * Lb, g.V), dtype=torch.uint8, device=DEV)

    class Step:
        lengths = [n + Lb for n in g.prompt]

    s, steps = Step(), 0
    while int(mask.sum()):
        block = g.normal(B * Lb, g.Hq + 2 * g.Hkv, g.d)
        s.q = g.append(block, block_seq, block_pos).view(B, Lb, g.Hq, g.d)
        s.out, s.lse = torch.empty_like(s.q), torch.empty((B, g.Hq, Lb), device=DEV)
        how = dict(lse=s.lse, mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=1 << 20, k_scale=g.scales[0], v_scale=g.scales[1])
        dlm.paged_attn(s.q, s.out, *g.pages, g.dev_table, g.kv_len, **how)
        dlm.lmhead_confidence(s.out.view(B * Lb, -1)[:, :g.Dh], g.w_vocab, conf, tok, workspace=ws)
        dlm.unmask_commit(conf, tok, g.x, mask, n_commit, remaining, x_pos0=0, rule=dlm.RULE_TOPK, k=2)
        torch.cuda.synchronize()
        # attention over what the pages now hold, in 64 bits
        k, v = (wide(x) * (1 if sc is None else wide(sc)[None, :, None, None]) for x, sc in zip(g.pages, g.scales))
        compare(s, *heads.paged_attention(wide(s.q), k, v, g.table, s.lengths))
        # and what they hold: the prompt's heads and this step's, from the projections
        table = wide(g.rope)
        for rows, sq, ps in ((prompt, seqs, pos), (block, block_seq, block_pos)):
            y = heads.head_map(wide(rows)[:, g.Hq:g.Hq + g.Hkv], wide(g.w[1]), 1e-6, table, ps, 0)
            got = k[g.table[sq, ps // g.page], :, ps % g.page]
            step = np.maximum(2.0 ** -4 * np.abs(y), 2.0 ** -10 * 0.06) if e4m3 else H * np.abs(y)
            assert (np.abs(got - y) <= step * (1 + H) + 256 * U * np.abs(y).max()).all()
        assert (n_commit == 2).all()
        steps += 1
    assert steps == Lb // 2 and (g.x[:, :Lb] == tok).sum() >= 2 * B


def test_training_forward_and_backward_through_attention():
    """d loss / d (queries, keys, weights) through rotation, norm and block-causal attention against 64-bit autograd of the definition.  The
    attention's own roundings (probabilities, their gradients and results in bf16) decide: 2^-7 of each tensor's norm, twice the half step of
    its three roundings' root mean square sum (sqrt(3) 2^-8 = 2^-7.2)."""
    rng = np.random.default_rng(11)
    T, Hq, Hkv, d, bs = 96, 4, 2, 64, 8
    n = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).to(BF16).to(DEV)
    qkv, d_out = n(T, Hq + 2 * Hkv, d), n(1, T, Hq, d)
    q, k, v = qkv.split([Hq, Hkv, Hkv], dim=1)
    w = [(1 + 0.2 * n(d).float()).to(BF16) for _ in range(2)]
    rope = torch.from_numpy(heads.angles(T, d).astype(np.float32)).to(DEV)
    pos = torch.arange(T, dtype=I32, device=DEV)
    how = dict(q_weight=w[0], k_weight=w[1], rope=rope, positions=pos)
    qr, kr = torch.empty((T, Hq, d), dtype=BF16, device=DEV), torch.empty((T, Hkv, d), dtype=BF16, device=DEV)
    dlm.qk_norm_rope(q, k, qr, kr, **how)
    batch = lambda t: t.transpose(0, 1)[None]                       # [1, H, T, d] view of [T, H, d]
    v_ = v.contiguous()
    out, lse = torch.empty((1, T, Hq, d), dtype=BF16, device=DEV), torch.empty((1, Hq, T), device=DEV)
    mask = dict(mask_mode=dlm.MASK_BLOCK_CAUSAL, block_size=bs)
    dlm.block_attn(qr[None], out, block=(batch(kr), batch(v_), 0), lse=lse, **mask)
    dq, dk, dv = torch.empty_like(qr), torch.empty_like(kr), torch.empty_like(v_)
    ws = torch.empty(dlm.block_attn_bwd_workspace_bytes(T, Hq), dtype=torch.uint8, device=DEV)
    dlm.block_attn_bwd(qr[None], out, d_out, lse, dq[None], block=(batch(kr), batch(v_), 0), d_block=(batch(dk), batch(dv)), workspace=ws, **mask)
    dw = [torch.empty(d, device=DEV) for _ in range(2)]
    ws = torch.empty(dlm.qk_norm_rope_bwd_workspace_bytes(T, Hq, Hkv, d), dtype=torch.uint8, device=DEV)
    dlm.qk_norm_rope_bwd(dq, dk, dq, dk, q=q, k=k, d_q_weight=dw[0], d_k_weight=dw[1], workspace=ws, **how)

    leaf = [t.detach().double().cpu().requires_grad_() for t in (q, k, v, w[0], w[1])]
    table = rope.double().cpu()

    def define(x, wt):
        x = x * wt / (x.pow(2).mean(-1, keepdim=True) + 1e-6).sqrt()
        c, s = table[:, None, :d // 2], table[:, None, d // 2:]
        return torch.cat([x[..., :d // 2] * c - x[..., d // 2:] * s, x[..., d // 2:] * c + x[..., :d // 2] * s], -1)

    y, z = define(leaf[0], leaf[3]), define(leaf[1], leaf[4]).repeat_interleave(Hq // Hkv, dim=1)
    s = torch.einsum("ihd,jhd->hij", y, z) / 8
    block = torch.arange(T) // bs
    p = s.masked_fill(block[None] > block[:, None], -float("inf")).softmax(-1)
    o = torch.einsum("hij,jhd->ihd", p, leaf[2].repeat_interleave(Hq // Hkv, dim=1))
    grads = torch.autograd.grad(o, leaf, d_out[0].double().cpu())
    for got, want in zip((dq, dk, dv, dw[0], dw[1]), grads):
        assert float((got.double().cpu() - want).norm() / want.norm()) <= 2.0 ** -7


def test_captured_steps_replay():
    """Append and attention of a step in one graph; replays with new heads and lengths in the same buffers, eager work in between."""
    g = Engine(False, seed=8)
    B = 3
    qkv, slots, pos = g.normal(B, g.Hq + 2 * g.Hkv, g.d), torch.zeros(B, dtype=I32, device=DEV), torch.zeros(B, dtype=I32, device=DEV)
    q_out, out = torch.empty((B, g.Hq, g.d), dtype=BF16, device=DEV), torch.empty((B, 1, g.Hq, g.d), dtype=BF16, device=DEV)
    kv_len = torch.ones(B, dtype=I32, device=DEV)
    table = torch.arange(3 * 256, dtype=I32, device=DEV).view(3, 256)
    pages = [torch.zeros((3 * 256, g.Hkv, g.page, g.d), dtype=BF16, device=DEV) for _ in range(2)]
    pages[0].copy_(g.normal(*pages[0].shape))
    pages[1].copy_(g.normal(*pages[1].shape))
    n = dlm.paged_attn_workspace_bytes(q_out[:, None], out, *pages, table, kv_len)
    assert n > 0
    ws = torch.empty(n, dtype=torch.uint8, device=DEV)

    def step(out_, pages_, ws_):
        q, k, v = qkv.split([g.Hq, g.Hkv, g.Hkv], dim=1)
        dlm.paged_append(k, v, *pages_, slots, q=q, q_out=q_out, q_weight=g.w[0], k_weight=g.w[1], rope=g.rope, positions=pos)
        dlm.paged_attn(q_out[:, None], out_, *pages_, table, kv_len, workspace=ws_)

    step(out, pages, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, pages, ws)
    for i in range(4):
        where = g.rng.integers(0, 4096, B)
        qkv.copy_(g.normal(*qkv.shape))
        pos.copy_(torch.from_numpy((where % 128).astype(np.int32)))
        slots.copy_(torch.from_numpy((where + 4096 * np.arange(B)).astype(np.int32)))
        kv_len.copy_(torch.from_numpy((where + 1).astype(np.int32)))
        eager_pages, eager_out = [x.clone() for x in pages], torch.empty_like(out)
        graph.replay()
        torch.cuda.synchronize()
        step(eager_out, eager_pages, torch.empty(n, dtype=torch.uint8, device=DEV))
        torch.cuda.synchronize()
        assert torch.equal(out, eager_out) and all(torch.equal(a, b) for a, b in zip(pages, eager_pages))
