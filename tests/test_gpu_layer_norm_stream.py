"""The residual stream through several layers, by the very lines that the README gives for a training step, against autograd
in 64 bits.  Gradients are held to 1e-5 of their norm: three layers of fp32 steps, each within a few 1e-7."""
import os
import re

import pytest
import torch

from paper_2101_11552_gb300 import build, tfg

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    build.build_library()


def readme_lines():
    """The forward and the backward of the layer norm as the README's training step has them."""
    with open(os.path.join(build.ROOT, "README.md")) as f:
        block = next(b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "tfg_layer_norm_backward(" in b)
    forward = next(line for line in block.splitlines() if "tfg.tfg_layer_norm(" in line)
    backward = re.search(r"^grad_stream.*?tfg_layer_norm_backward\(.*?\)\n", block, re.S | re.M).group(0)
    return compile(forward.strip(), "forward", "exec"), compile(backward, "backward", "exec")


@pytest.mark.parametrize("f", [64, 37])
def test_three_layers_of_a_stream(f):
    forward, backward = readme_lines()
    n_rows, layers = 200, 3
    gen = torch.Generator(device="cuda").manual_seed(f)
    draw = lambda *shape: torch.randn(*shape, device="cuda", generator=gen)
    start, branches, outs = draw(n_rows, f), [draw(n_rows, f) for _ in range(layers)], [draw(n_rows, f) for _ in range(layers)]
    gammas, betas = [1 + 0.1 * draw(f) for _ in range(layers)], [0.1 * draw(f) for _ in range(layers)]

    leaves = [t.double().requires_grad_() for t in (start, *branches, *gammas, *betas)]
    stream, loss = leaves[0], 0.0
    for k in range(layers):
        stream = stream + leaves[1 + k]
        normed = (stream - stream.mean(1, keepdim=True)) / (stream.var(1, unbiased=False, keepdim=True) + 1e-5).sqrt()
        loss = loss + ((normed * leaves[1 + layers + k] + leaves[1 + 2 * layers + k]) * outs[k].double()).sum()
    want = torch.autograd.grad(loss + (stream * outs[0].double()).sum(), leaves)

    kept, stream = [], start.clone()
    for k in range(layers):
        here = dict(tfg=tfg, branch=branches[k], gamma=gammas[k], beta=betas[k], stream=stream)
        exec(forward, here)
        kept.append(here)
        stream = here["n"].sum
    got, grad_stream = [None] * len(want), outs[0].clone()
    for k in reversed(range(layers)):
        here = dict(kept[k], grad_out=outs[k], grad_stream=grad_stream)
        exec(backward, here)
        grad_stream = here["grad_stream"]
        got[1 + k], got[1 + layers + k], got[1 + 2 * layers + k] = grad_stream.clone(), here["grad_gamma"], here["grad_beta"]
    got[0] = grad_stream
    for a, b in zip(got, want):
        assert float((a.double() - b).norm()) <= 1e-5 * float(b.norm())


@pytest.mark.parametrize("f", [64, 37, 3001])
def test_where_values_that_are_no_numbers_go(f):
    """As the header says: a row of the sum that holds one reaches its own row of grad_s and grad_gamma, not grad_beta; what
    grad_out holds of them reaches its row and both sums.  Deviations beyond fp32's squares give rstd 0."""
    gen = torch.Generator(device="cuda").manual_seed(f)
    x, g = (torch.randn(40, f, device="cuda", generator=gen) for _ in range(2))
    gamma, beta = torch.rand(f, device="cuda", generator=gen), torch.rand(f, device="cuda", generator=gen)
    x[4, f // 2] = float("nan")
    x[9, 1] = 1e25
    r = tfg.tfg_layer_norm(x, gamma, beta)
    assert float(r.rstd[9]) == 0.0 and torch.equal(r.out[9], beta) and bool(torch.isnan(r.out[4]).all())
    gx, gg, gb = tfg.tfg_layer_norm_backward(x, gamma, r.mean, r.rstd, g)
    rest = [i for i in range(40) if i != 4]
    assert bool(torch.isnan(gx[4]).all()) and bool(torch.isfinite(gx[rest]).all())
    assert bool(torch.isnan(gg).all()) and bool(torch.isfinite(gb).all())
    g[11, 2] = float("inf")
    x[4] = 1.0
    r = tfg.tfg_layer_norm(x, gamma, beta)
    gx, gg, gb = tfg.tfg_layer_norm_backward(x, gamma, r.mean, r.rstd, g)
    rest = [i for i in range(40) if i != 11]
    assert not bool(torch.isfinite(gx[11]).any()) and bool(torch.isfinite(gx[rest]).all())
    assert not bool(torch.isfinite(gg[2])) and not bool(torch.isfinite(gb[2]))
    others = [c for c in range(f) if c != 2]
    assert bool(torch.isfinite(gb[others]).all())
