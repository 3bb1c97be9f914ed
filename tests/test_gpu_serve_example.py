"""The serving example: its graph steps against the same steps run eagerly, and against the layers computed with torch in
fp32 from the unpacked weights and what the cache holds."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("serve_layers", os.path.join(ROOT, "examples", "serve_layers.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def _small(m, requests=3):
    import torch

    cfg = m.Config(hidden=256, ffn=512, heads=4, kv_heads=2, head_dim=64, layers=2, page=16, dtype=torch.float16)
    return m.Server(cfg, requests, 80)


def _prompts(server, lens):
    import torch

    g = torch.Generator(device="cuda").manual_seed(7)
    new = torch.tensor(lens, dtype=torch.int32, device="cuda")
    x = torch.randn(sum(lens), server.cfg.hidden, generator=g, device="cuda").to(server.cfg.dtype)
    y = server.step(x, new, max(lens))
    return x, y[new.cumsum(0) - 1]


def test_graph_steps_equal_eager_steps():
    import torch

    m = _example()
    a, b = _small(m), _small(m)
    (_, ya), (_, yb) = _prompts(a, [30, 1, 17]), _prompts(b, [30, 1, 17])
    assert torch.equal(ya, yb)
    graph, x, out = a.capture()
    x.copy_(ya)
    one = torch.ones(3, dtype=torch.int32, device="cuda")
    for i in range(20):
        graph.replay()
        yb = b.step(yb, one, 1)
        torch.cuda.synchronize()
        assert torch.equal(out, yb), i
        x.copy_(out)
    assert b.lens.tolist() == [50, 21, 37] and a.lens.tolist() == [50, 21, 37]


def test_a_prompt_against_the_plain_layers():
    """Against fp32 torch over the unpacked weights and, for attention, the cache's own keys and values.  Activations are
    rounded to fp16 some ten times a layer (2^-11 each, of terms that add up over two layers): 2% of the largest output
    is far more than that and far less than any wrong head, position or weight."""
    import torch

    import paper_2405_03594_amd as spl

    m = _example()
    s = _small(m, 1)
    n = 45
    x, _ = _prompts(s, [n])
    t, slots = torch.arange(n, device="cuda"), None
    slots = (s.table[0, t // 16] * 16 + t % 16).int()
    y = x.float()
    cfg = s.cfg
    for layer in s.layers:
        w = {k: spl.unpack(getattr(layer, k)).float() for k in ("q", "o", "gate", "up", "down")}
        z = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + cfg.eps)
        q = (z @ w["q"].T).view(n, cfg.heads, cfg.head_dim)
        q = q * torch.rsqrt(q.square().mean(-1, keepdim=True) + cfg.eps)
        c, si = s.rope[:n, None, :, 0], s.rope[:n, None, :, 1]
        a, b = q.split(cfg.head_dim // 2, -1)
        q = torch.cat((a * c - b * si, b * c + a * si), -1)
        k, v = (u.float().repeat_interleave(cfg.heads // cfg.kv_heads, 1) for u in spl.cache_read(layer.cache, slots))
        p = torch.einsum("thd,uhd->htu", q, k) * cfg.head_dim ** -0.5
        p = p.masked_fill(t[None, None] > t[None, :, None], float("-inf")).softmax(-1)
        y = y + torch.einsum("htu,uhd->thd", p, v).reshape(n, -1) @ w["o"].T
        z = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + cfg.eps)
        y = y + (torch.nn.functional.silu(z @ w["gate"].T) * (z @ w["up"].T)) @ w["down"].T
    again = _small(m, 1)
    got = again.step(x, torch.tensor([n], dtype=torch.int32, device="cuda"), n)
    torch.cuda.synchronize()
    assert (got.float() - y).abs().max() < 0.02 * y.abs().max()


def test_the_command_runs(capsys):
    _example().main(["--layers", "1", "--requests", "2", "--prompt", "20", "--steps", "3", "--hidden", "256", "--ffn",
                     "512", "--heads", "4", "--kv-heads", "2", "--head-dim", "64"])
    assert "token steps" in capsys.readouterr().out
