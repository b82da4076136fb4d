"""README's recipe of a training step through a token model's ends, as it stands there, with blocks of a program's own between them: its
gradients against automatic differentiation in float64."""
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _recipe():
    text = open(os.path.join(ROOT, "README.md")).read()
    return [b for b in re.findall(r"```python\n(.*?)```", text, re.S) if "sgd_kernel_embedding_grad" in b]


def test_gradients_of_the_recipe():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2609_29505_gb300 import binding, build
    build.build()
    torch.backends.cuda.matmul.allow_tf32 = False
    V, d, rows, k = 300, 64, 90, 6
    gen = torch.Generator().manual_seed(6)

    def r(*s):
        return torch.randn(*s, generator=gen).cuda()
    mix = r(d, d) / d ** 0.5
    a = dict(binding=binding, table=r(V, d), gain=(1 + 0.1 * r(d)).bfloat16(), head=r(V, d) / d ** 0.5, x=torch.empty(rows, d, device="cuda"),
             n=torch.empty(rows, d, device="cuda", dtype=torch.float16), loss=torch.empty(rows, device="cuda"), dz=torch.empty(rows, V, device="cuda"),
             dh=torch.empty(rows, d, device="cuda"), dgain=torch.empty(d, device="cuda"), dtable=torch.empty(V, d, device="cuda"),
             ids=torch.randint(0, V, (rows,), generator=gen, dtype=torch.int32).cuda(),
             top=torch.stack([torch.randperm(V, generator=gen)[:k] for _ in range(rows)]).int().cuda(),
             logq=torch.log_softmax(r(rows, k + 1), 1)[:, :k].contiguous(), blocks=lambda x: x + x @ mix, blocks_backward=lambda dh: dh + dh @ mix.T)
    [code] = _recipe()
    table, gain, head = (a[n].double().requires_grad_() for n in ("table", "gain", "head"))
    x = table[a["ids"].long()]
    h = x + x @ mix.double()
    z = h / torch.sqrt(h.pow(2).mean(1, keepdim=True) + 1e-6) * gain @ head.T
    lp, q = torch.log_softmax(z, 1), a["logq"].double().exp()
    inside = torch.zeros_like(z, dtype=torch.bool).scatter_(1, a["top"].long(), True)
    qt, lpt = 1 - q.sum(1), torch.logsumexp(lp.masked_fill(inside, -torch.inf), 1)
    loss = (q * (a["logq"].double() - torch.gather(lp, 1, a["top"].long()))).sum(1) + qt * (qt.log() - lpt)
    loss.sum().backward()
    exec(code, a)
    # The normed rows are fp16 (2^-12 of them at most), the logits, sums of d terms, off by as much of their terms, and so p: ten times 2^-11 of the
    # gradients' norms, as in test_gpu_ends_run.py; the products are fp32.
    assert (a["loss"].double() - loss.detach()).abs().max() <= 10 * 2.0 ** -11
    for got, want in ((a["dtable"], table.grad), (a["dgain"], gain.grad), (a["dhead"], head.grad)):
        assert (got.double() - want).norm() <= 10 * 2.0 ** -11 * want.norm()
