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


MEMORY = ("global_", "scratch_", "flat_", "buffer_", "ds_")


def registers(operands, kind):
    """Numbers of the registers of a kind ('a' or 'v') that stand in a list of operands."""
    out = set()
    for one, first, last in re.findall(kind + r"(?:(\d+)\b|\[(\d+):(\d+)\])", re.sub(r"\b0x\w+", "", operands)):
        out |= {int(one)} if one else set(range(int(first), int(last) + 1))
    return out


def parts(x):
    name, _, rest = x.partition(" ")
    return name, [o.strip() for o in re.split(r",\s*(?![^\[]*\])", rest.split(";")[0])]


def violations(body):
    """What comes too near to a product: memory instructions that read or write accumulation registers, and ordinary instructions that
    write its factors (2 before) or the lanes that take part (4 before)."""
    labels = {x.split(":")[0]: n for n, x in enumerate(body) if x.startswith(".LBB")}

    def follow(n):
        x = body[n]
        if x.startswith("s_endpgm"):
            return []
        to = [labels[x.split()[1]]] if x.startswith(("s_branch", "s_cbranch")) else []
        return to if x.startswith("s_branch") else to + [n + 1]

    is_product = lambda x: x.startswith("v_mfma") and " a[" in x.split(",")[0]  # noqa: E731
    on_sums = lambda x: x.startswith(MEMORY) and bool(registers(x.partition(" ")[2], r"\ba"))  # noqa: E731
    found = []
    for n, x in enumerate(body):
        if is_product(x):
            y = near(body, follow, n, on_sums, 18)
            found += [(x, y)] if y else []
        elif on_sums(x) and "load" in x.split()[0] + "load" * x.startswith("ds_read"):
            y = near(body, follow, n, is_product, 6)
            found += [(x, y)] if y else []
        elif x.startswith("v_") and not x.startswith(("v_mfma", "v_accvgpr_write", "v_accvgpr_mov")):
            name, operands = parts(x)
            if name.startswith("v_cmpx"):
                y = near(body, follow, n, is_product, 3)
                found += [(x, y)] if y else []
            written = registers(operands[0], r"\bv")
            reads = lambda y: is_product(y) and bool(written & registers(" ".join(parts(y)[1][1:3]), r"\bv"))  # noqa: E731
            y = near(body, follow, n, reads, 1) if written else None
            found += [(x, y)] if y else []
    return found


def bodies(source, out):
    flags = [f for f in build.FLAGS if f not in ("-fPIC", "-shared")]
    subprocess.check_call([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *flags, "-S", "--offload-device-only", "-o", out,
                           os.path.join(build.CSRC, source)], stderr=subprocess.DEVNULL)
    text = open(out).read()
    return {m.group(1): [x.strip() for x in text[m.end():text.index(".Lfunc_end", m.end())].split("\n")]
            for m in re.finditer(r"^(_ZN2dc\w+):", text, re.M)}


@pytest.mark.parametrize("source", ["head.hip", "head_grad.hip"])
def test_memory_instructions_and_factors_keep_their_distance(source, tmp_path):
    """The compiler may store sums from their registers, spill them there and load them, without another instruction between."""
    every = bodies(source, str(tmp_path / "code.s"))
    kernels = {n: b for n, b in every.items() if KERNELS.search(n)}
    assert len(kernels) >= 12
    for name, body in kernels.items():
        assert not violations(body), (name, violations(body)[:3])
    if source == "head.hip":                                  # (that such stores are known when they are met: the few rows' kernels have some)
        assert any(x.startswith("global_store") and registers(x, r"\ba") for n, b in every.items() if "head_few" in n for x in b)


def test_the_search_finds_what_comes_too_near():
    product = "v_mfma_f32_16x16x32_bf16 a[0:3], v[4:7], v[8:11], a[0:3]"
    idle = ["s_nop 15", "s_nop 15"]
    store, load, spill = "global_store_dwordx4 v[0:1], a[0:3], off", "global_load_dwordx4 a[4:7], v[0:1], off", "scratch_store_dwordx4 off, a[28:31], off"
    end = ["s_endpgm"]
    for x in (store, spill, load, "ds_write_b128 v0, a[0:3]", "ds_read_b128 a[0:3], v0"):
        assert violations([product, x, *end]) and violations([product, *["v_nop"] * 17, x, *end])
        assert not violations([product, *idle, x, *end])
        assert violations([".LBB0_1:", x, "s_nop 0", product, *idle, "s_cbranch_scc1 .LBB0_1", *end]) == \
            ([] if "store" in x or "write" in x else [(x, product)])
    loop = [".LBB0_1:", store, *idle, product, "s_cbranch_scc1 .LBB0_1", *end]      # around a loop
    assert violations(loop)
    for x in ("v_mov_b32_e32 v5, v0", "v_cndmask_b32_e32 v10, v0, v1, vcc", "v_cvt_pk_bf16_f32 v4, v0, v1"):
        assert violations([x, product, *end]) and violations([x, "s_nop 0", product, *end])
        assert not violations([x, "s_nop 0", "s_nop 0", product, *end])
    assert not violations(["v_mov_b32_e32 v12, v5", product, *end])
