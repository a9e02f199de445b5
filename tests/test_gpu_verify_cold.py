"""Verification at temperatures so low that logits over the temperature pass what a 64-bit
log-sum-exp resolves: probabilities are those of the draws, ties at the top among them, and every
decision equals the float64 oracle's.  Uniforms lie 5e-5 at least from the border of a decision
between ties (n equal entries weigh 1 / n each)."""
import numpy as np
import pytest
import torch

import test_gpu_truncation as base
from oracle import truncation as tr
from paper_2606_26744_amd import hdf

pytestmark = pytest.mark.gpu
DEV = "cuda"
COLD = [1e-3, 1e-6, 1e-9, 1e-14, 1e-30, 1e-42]


def _rows(n, B, V, seed, dd, td):
    """Draft and target rows whose greatest logits are shared by some tokens: none, some or all of
    them the same tokens on both sides."""
    g = torch.Generator().manual_seed(seed)
    z = torch.randn(n * B, V, generator=g) * 2
    t = torch.randn(n, B, V, generator=g) * 2
    for s in range(n):
        for i in range(B):
            top = torch.randperm(V, generator=g)[:5]
            m = float(torch.randint(9, 20, (1,), generator=g))
            kind = (s + i) % 4
            if i + 1 < B:
                z[s * B + i + 1, top[:[1, 2, 3, 1][kind]]] = m
            t[s, i, top[[0, 0, 1, 0][kind]:[1, 3, 4, 2][kind]]] = m + 0.25 * kind
    return z.to(dd).to(DEV), t.to(td).to(DEV)


def _uniforms(n, B, seed):
    """Away from every quotient of two numbers up to 4."""
    g = torch.Generator().manual_seed(seed)
    return ((torch.randint(0, 500, (n, B), generator=g) + 0.37) / 500).to(DEV)


@pytest.mark.parametrize("dd,td", [(torch.float32, torch.float32), (torch.bfloat16, torch.float32),
                                   (torch.float32, torch.bfloat16)])
@pytest.mark.parametrize("T", COLD)
def test_cold_verification(T, dd, td):
    n, B, V = 8, 6, 3001
    accepted = []
    for seed, cuts in ((1, {}), (2, dict(top_p=0.9)), (3, dict(top_k=2)), (4, dict(min_p=0.5))):
        kw = dict(temperature=T, **cuts)
        z, t = _rows(n, B, V, seed, dd, td)
        tok, cut = hdf.sample_truncated(z, base._u(n * B, seed + 9), rows_per_seq=B, **kw)
        accepted += base._check_verify(n, B, V, z, t, tok, cut, _uniforms(n, B, seed), kw)
    assert min(accepted) < max(accepted)


def test_a_temperature_a_sequence():
    n, B, V = len(COLD) + 2, 5, 4099
    z, t = _rows(n, B, V, 7, torch.float32, torch.float32)
    kw = dict(temperature=torch.tensor(COLD + [0.0, 1.0], device=DEV))
    tok, cut = hdf.sample_truncated(z, base._u(n * B, 3), rows_per_seq=B, **kw)
    base._check_verify(n, B, V, z, t, tok, cut, _uniforms(n, B, 8), kw)


@pytest.mark.parametrize("T", [1e-9, 1e-30])
def test_the_same_rows_accept_everything(T):
    n, B, V = 3, 70, 2003
    z, _ = _rows(n, B, V, 5, torch.float32, torch.float32)
    t = torch.empty(n, B, V, device=DEV)
    t[:, :B - 1] = z.view(n, B, V)[:, 1:]
    t[:, B - 1] = z.view(n, B, V)[:, 0]
    kw = dict(temperature=T)
    tok, cut = hdf.sample_truncated(z, base._u(n * B, 3), rows_per_seq=B, **kw)
    u = torch.full((n, B), 1 - 2.0 ** -24, device=DEV)
    u[:, B - 1] = 0.3
    acc = base._check_verify(n, B, V, z, t, tok, cut, u, kw)
    assert acc == [B - 1] * n
    # A draft that is no token leaves no residual: the next token comes from the target's own.
    tok[B + 4] = V
    acc = base._check_verify(n, B, V, z, t, tok, cut, u, kw)
    assert acc == [B - 1, 3, B - 1]


@pytest.mark.parametrize("scale", [1e9, 1e30])
def test_large_logits(scale):
    """The same at T = 1 of logits that are large themselves, masked rows and entries among them."""
    n, B, V = 6, 5, 1500
    z, t = _rows(n, B, V, 11, torch.float32, torch.float32)
    z, t = z * scale, t * scale
    z[2, ::2] = -np.inf
    t[1, 1] = -np.inf
    t[2, :, 7:900] = float("nan")
    z[3 * B + 1] = -np.inf
    tok, cut = hdf.sample_truncated(z, base._u(n * B, 2), rows_per_seq=B)
    base._check_verify(n, B, V, z, t, tok, cut, _uniforms(n, B, 4), {})


def test_cold_verification_replays():
    """Captured and replayed, over a workspace of arbitrary contents."""
    n, B, V = 4, 5, 3001
    kw = dict(temperature=1e-9)
    ws = torch.full((hdf.lib().hdf_accept_truncated_workspace(n, B - 1, V, 0),), 255, dtype=torch.uint8,
                    device=DEV)
    z, t = _rows(n, B, V, 1, torch.float32, torch.float32)
    tok, cut = hdf.sample_truncated(z, base._u(n * B, 1), rows_per_seq=B, **kw)
    u = _uniforms(n, B, 1)
    out = tuple(torch.zeros(m, dtype=torch.int32, device=DEV) for m in (n, n, n + 1, n * B))

    def call():
        return hdf.accept_truncated(tok[1:], z[1:], tuple(x[1:] for x in cut), t, u, K=B - 1,
                                    draft_stride=B, out=out, ws=ws, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(1, 5):
        z2, t2 = _rows(n, B, V, seed, torch.float32, torch.float32)
        tok2, cut2 = hdf.sample_truncated(z2, base._u(n * B, seed), rows_per_seq=B, **kw)
        z.copy_(z2), t.copy_(t2), tok.copy_(tok2), u.copy_(_uniforms(n, B, seed))
        for a, b in zip(cut, cut2):
            a.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in out]
        for x in out:
            x.zero_()
        call()
        torch.cuda.synchronize()
        live = int(out[2][-1])
        assert all(torch.equal(a[:live], b[:live]) for a, b in zip(got, out)), seed
