"""The cases that the point-wise product's accuracy is measured at reach every kernel built for it, and its bounds lie below what a lost term costs."""
import re

import pytest
import torch

from tests import block_reference as ref
from tests import launches, product_accuracy as pa
from tests.test_abi_host import kernel_notes, lib  # noqa: F401


def test_cases_reach_every_kernel(lib, tmp_path):  # noqa: F811
    program = launches.build(tmp_path)
    if program is None:
        pytest.skip("no hipcc")
    built = {k[0] for k in kernel_notes() if re.search("product_(thin_|weights_)?kernel|strip_(back_)?kernel", k[0])}
    acts = {"none": 0, "silu": 2}
    calls = [(name, *case[:-1], acts[case[-1]], flag) for case in pa.CASES for name in ("pointwise_forward", "pointwise_backward") for flag in (0, 1)]
    reached = {l.kernel for _, made in launches.ask(program, calls) for l in made}
    assert len(built) > 130 and built <= reached, built - reached


def test_bounds_notice_a_lost_term():
    assert all(bar < 0.8 * pa.LOST for case in pa.CASES for bar in pa.bars(case).values())
    for K, M in ((16, 30), (64, 65), (300, 130)):
        g = torch.Generator().manual_seed(K)
        x, w, b, go = (torch.randn(*s, generator=g) for s in ((K, 4000), (M, K), (M, 1), (M, 4000)))
        w = w * K ** -0.5
        X, W, G = x.double(), w.double(), go.double()
        pre = W @ X + b.double()
        gp = G * ref.slope("silu", pre)
        lost = {"out": [(W @ pa.two_of_three(x) + b.double(), pre), (pa.two_of_three(w) @ X + b.double(), pre)],
                "grad_x": [(pa.two_of_three(w).t() @ gp, W.t() @ gp), (W.t() @ pa.two_of_three(gp.float()), W.t() @ gp)],
                "grad_w": [(pa.two_of_three(gp.float()) @ X.t(), gp @ X.t()), (gp @ pa.two_of_three(x).t(), gp @ X.t())]}
        for other in (W @ pa.two_of_three(x) + b.double(), pa.two_of_three(w) @ X + b.double()):
            g2 = G * ref.slope("silu", other)
            lost["grad_x"].append((W.t() @ g2, W.t() @ gp)), lost["grad_w"].append((g2 @ X.t(), gp @ X.t()))
        for name, pairs in lost.items():
            assert all(pa.off(*pair) > pa.LOST for pair in pairs), (K, M, name, [pa.off(*pair) for pair in pairs])
        # bf16 results: with one term less many more are rounded the other way
        xb, gb = x.bfloat16().double(), gp.float()
        for got, want in ((pa.one_of_two(w) @ xb, W @ xb), (pa.one_of_two(w).t() @ gp, W.t() @ gp), (W.t() @ pa.one_of_two(gb), W.t() @ gp)):
            assert (got.bfloat16() != want.bfloat16()).double().mean() > 10 * pa.OTHERS
