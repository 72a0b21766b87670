"""The 64-bit definitions of the sequence operators against torch's own operators and automatic derivatives on the CPU, and
the checks of arguments that need no GPU."""

import numpy as np
import pytest
import torch

from oracle import sequence as ref


def leaf(*shape, seed=0, scale=1.0):
    return torch.from_numpy(np.random.default_rng(seed + sum(shape)).standard_normal(shape) * scale).requires_grad_()


def near(a, b):
    assert np.allclose(a, b.detach().numpy(), rtol=1e-10, atol=1e-12)


@pytest.mark.parametrize("n,d,k,act", [(9, 4, 3, True), (2, 3, 5, True), (6, 2, 1, False), (1, 5, 4, True)])
def test_convolution(n, d, k, act):
    x, w, b, st = leaf(n, d), leaf(d, k, seed=1), leaf(d, seed=2), leaf(k - 1, d, seed=3)
    line = torch.cat([st, x])
    pre = torch.nn.functional.conv1d(line.t()[None], w[:, None], b, groups=d)[0].t()
    y = torch.nn.functional.silu(pre) if act else pre
    dy, df = leaf(n, d, seed=4).detach(), leaf(k - 1, d, seed=5).detach()
    ((y * dy).sum() + (line[n:] * df).sum()).backward()
    args = [v.detach().numpy() for v in (x, w, b, st)]
    got, last, _ = ref.conv_causal(*args, act)
    near(got, y), near(last, line[n:])
    g = ref.conv_causal_backward(dy.numpy(), *args, act, df.numpy())
    near(g["dx"], x.grad), near(g["dw"], w.grad), near(g["db"], b.grad)
    if k > 1:
        near(g["dstate"], st.grad)


@pytest.mark.parametrize("n,d,states,groups,plus", [(7, 4, 3, 2, True), (1, 2, 16, 1, True), (5, 3, 2, 1, False)])
def test_scan(n, d, states, groups, plus):
    u, delta, z = leaf(n, d), leaf(n, d, seed=1, scale=0.5), leaf(n, d, seed=2)
    B, C, A = leaf(n, groups, states, seed=3), leaf(n, groups, states, seed=4), leaf(d, states, seed=5)
    D, bias, st = leaf(d, seed=6), leaf(d, seed=7), leaf(d, states, seed=8)
    dl = delta + bias
    dl = torch.nn.functional.softplus(dl) if plus else dl
    h, ys = st, []
    for t in range(n):
        b, c = (v[t].repeat_interleave(d // groups, 0) for v in (B, C))
        h = torch.exp(dl[t][:, None] * A) * h + (dl[t] * u[t])[:, None] * b
        ys.append((h * c).sum(1) + D * u[t])
    y = torch.stack(ys) * torch.nn.functional.silu(z)
    dy, df = leaf(n, d, seed=9).detach(), leaf(d, states, seed=10).detach()
    ((y * dy).sum() + (h * df).sum()).backward()
    args = dict(u=u, delta=delta, A=A, B=B, C=C, D=D, z=z, bias=bias, state=st)
    args = dict({k: v.detach().numpy() for k, v in args.items()}, plus=plus)
    f = ref.scan(**args)
    near(f["y"], y), near(f["final"], h)
    g = ref.scan_backward(dy.numpy(), **args, dfinal=df.numpy())
    for name, v in (("du", u), ("dd", delta), ("dz", z), ("dA", A), ("dB", B), ("dC", C), ("dD", D), ("dbias", bias), ("dstate", st)):
        near(g[name], v.grad)
        assert (g[name + "_mag"] >= np.abs(g[name]) * 0.999999).all()


def test_group_norm():
    x, w, b = leaf(3, 5, 12), leaf(12, seed=1), leaf(12, seed=2)
    pre = torch.nn.functional.group_norm(x.transpose(1, 2), 4, w, b, 1e-5).transpose(1, 2)
    y = torch.nn.functional.silu(pre)
    dy = leaf(3, 5, 12, seed=3).detach()
    (y * dy).sum().backward()
    args = [v.detach().numpy() for v in (x,)] + [4] + [v.detach().numpy() for v in (w, b)]
    near(ref.groupnorm(*args, 1e-5, True)[0], y)
    g = ref.groupnorm_backward(dy.numpy(), *args, 1e-5, True)
    near(g["dx"], x.grad), near(g["dw"], w.grad), near(g["db"], b.grad)


@pytest.fixture(scope="module")
def seq():
    from paper_2010_15884_b200 import build
    build.build()
    from paper_2010_15884_b200 import sequence
    sequence._library()
    return sequence


ENTRIES = ["sysconv1d_causal", "sysconv1d_causal_backward", "sysscan", "sysscan_backward", "sysgroupnorm", "sysgroupnorm_backward"]


def test_null_and_empty_descriptors_are_refused(seq):
    lib = seq._library()
    sizes = {"sysconv1d_causal": seq._CAUSAL, "sysconv1d_causal_step": seq._CAUSAL_STEP, "sysscan": seq._SCAN,
             "sysscan_step": seq._SCAN_STEP, "sysgroupnorm": seq._NORM}
    for name in ENTRIES + ["sysconv1d_causal_step", "sysscan_step"]:
        form = sizes[name.replace("_backward", "")]
        assert getattr(lib, name)(None, None) == 1
        assert getattr(lib, name)(bytes(form.size), None) == 1
    for name in ("sysconv1d_causal_backward_workspace_bytes", "sysscan_saved_blocks", "sysscan_workspace_bytes",
                 "sysscan_backward_workspace_bytes", "sysgroupnorm_workspace_bytes", "sysgroupnorm_backward_workspace_bytes"):
        assert getattr(lib, name)(None) == -1


def test_descriptors_out_of_range(seq):
    """Each member in turn made wrong in a descriptor that would otherwise be taken (pointers are never followed)."""
    lib, p = seq._library(), 4096
    tok = (p, 80, 8)
    good = [2, 10, 20, 0, 0, 8, 4, 1, 1, 1, *tok, *tok, 0, 0, 0, p, p, p, 0, 0, 0, 0, 0, 0, 0]
    for at, value, status in ((0, 0, 1), (1, -1, 1), (5, 0, 1), (6, 0, 1), (7, 3, 1), (7, -1, 1), (8, 2, 1), (9, 2, 1), (10, 0, 1),
                              (12, -8, 1), (13, 0, 1), (14, 7, 1), (15, 7, 1), (19, 0, 1), (6, 9, 2), (0, 1 << 31, 2), (5, 1 << 29, 2)):
        bad = list(good)
        bad[at] = value
        if at == 5 and value > 8:
            bad[14] = bad[15] = bad[11] = bad[12] = value
        assert lib.sysconv1d_causal(seq._CAUSAL.pack(*bad), None) == status, (at, value)
    # group norm: batch, space, channels, groups, type, activation, eps
    good = [2, 10, 8, 2, 1, 1, 1e-5, *tok, *tok, 0, 0, 0, 0, 0, 0, p, p, 0, 0, 0, 0, 0, 0]
    for at, value in ((0, 0), (1, 0), (2, 9), (3, 0), (3, 3), (4, 9), (5, 5), (6, -1e-5), (6, float("nan")), (7, 0), (10, 0), (12, 4)):
        bad = list(good)
        bad[at] = value
        assert lib.sysgroupnorm(seq._NORM.pack(*bad), None) == 1, (at, value)
    tn = (p, 160, 16)
    good = [2, 10, 20, 0, 0, 8, 16, 1, 1, 1, *tok, *tok, *tok, *tn, *tn, *tok, p, p, p, p, 0, 0, *[0] * 18, 0, 0, 0, 0, 0, 0, 0]
    for at, value, status in ((0, 0, 1), (5, 0, 1), (6, 0, 1), (7, 3, 1), (8, 4, 1), (10, 0, 1), (13, 0, 1), (19, 0, 1), (22, 0, 1),
                              (25, 0, 1), (27, 7, 1), (28, 0, 1), (6, 129, 2), (0, 65536, 2)):
        bad = list(good)
        bad[at] = value
        assert lib.sysscan(seq._SCAN.pack(*bad), None) == status, (at, value)


def test_workspace_and_saved_sizes(seq):
    lib, p = seq._library(), 4096

    def scan(r, n, d, states, total=None):
        off = (0, 0) if total is None else (p, 0)
        return seq._SCAN.pack(r, n, total or 0, *off, d, states, 1, 1, 1, *(p, n * d, d) * 3, *(p, n * states, states) * 2,
                              p, n * d, d, p, p, p, p, 0, 0, *[0] * 18, 0, 0, 0, 0, 0, 0, 0)

    assert lib.sysscan_saved_blocks(scan(3, 33, 8, 16)) == 9
    assert lib.sysscan_saved_blocks(scan(3, 33, 8, 16, total=40)) == 5
    assert lib.sysscan_workspace_bytes(scan(8, 2048, 4096, 16)) == 0                 # enough channels: one pass
    assert lib.sysscan_workspace_bytes(scan(1, 8192, 64, 16)) > 0                    # split over tokens
    assert lib.sysscan_workspace_bytes(scan(1, 100, 64, 16)) == 0                    # too short to split


def test_tensors_on_the_cpu_are_refused(seq):
    x, w = torch.zeros(1, 4, 8), torch.zeros(8, 4)
    for call in (lambda: seq.conv1d_causal(x, w), lambda: seq.groupnorm(x, 2),
                 lambda: seq.state_scan(x, x, torch.zeros(8, 16), torch.zeros(1, 4, 16), torch.zeros(1, 4, 16))):
        with pytest.raises(seq.SysconvError):
            call()
