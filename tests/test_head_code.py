"""What the compiler makes of the head's products: the accumulation registers' distances.

The products are written as instructions that the compiler does not know for matrix products, so it does not keep the distance that
other accesses of their sums need (a read at least 18 instructions behind, whatever the product's length; a write at least 2 before):
the source does, with 32 idle cycles on either side.  This follows every way through the kernels' code and looks whether a compiler
has moved one across.
"""
import os
import re
import subprocess

import pytest

from paper_2507_13833_amd import build

KERNELS = re.compile(r"head_(stat|logits|piece|hidden|weight)_kernel")


def near(body, follow, start, wanted, limit):
    """The first wanted instruction within `limit` of start on some way without idle cycles."""
    seen, todo = {}, [(n, 0) for n in follow(start)]
    while todo:
        n, d = todo.pop()
        if n >= len(body) or seen.get(n, limit + 1) <= d:
            continue
        seen[n] = d
        x = body[n]
        if x.startswith("s_nop 15"):
            continue
        if wanted(x):
            return x
        if d < limit:
            todo += [(m, d + bool(x and x[0] not in ";./")) for m in follow(n)]
    return None


@pytest.mark.parametrize("source", ["head.hip", "head_grad.hip"])
def test_products_keep_their_distance(source, tmp_path):
    flags = [f for f in build.FLAGS if f not in ("-fPIC", "-shared")]
    out = str(tmp_path / "code.s")
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-S", "--offload-device-only", "-o", out,
                           os.path.join(build.CSRC, source)], stderr=subprocess.DEVNULL)
    text = open(out).read()
    kernels = [m for m in re.finditer(r"^(_ZN2dc\w+):", text, re.M) if KERNELS.search(m.group(1))]
    assert len(kernels) >= 12
    product = lambda x: x.startswith("v_mfma") and " a[" in x.split(",")[0]  # noqa: E731
    for m in kernels:
        body = [x.strip() for x in text[m.end():text.index(".Lfunc_end", m.end())].split("\n")]
        labels = {x.split(":")[0]: n for n, x in enumerate(body) if x.startswith(".LBB")}

        def follow(n):
            x = body[n]
            if x.startswith("s_endpgm"):
                return []
            to = [labels[x.split()[1]]] if x.startswith(("s_branch", "s_cbranch")) else []
            return to if x.startswith("s_branch") else to + [n + 1]

        assert any(product(x) for x in body), m.group(1)
        for n, x in enumerate(body):
            if product(x):
                assert near(body, follow, n, lambda y: y.startswith("v_accvgpr"), 18) is None, m.group(1)
            elif x.startswith(("v_accvgpr_write", "v_accvgpr_mov")):
                assert near(body, follow, n, product, 6) is None, m.group(1)
