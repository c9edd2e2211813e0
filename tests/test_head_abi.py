"""Refusals of the head's log-probabilities and of the residual norm: what is turned down before anything touches a GPU."""
import ctypes as C
import math
import os
import re

import pytest

from paper_2507_13833_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000                                                   # never dereferenced: every call below fails validation first
WS = 1 << 45


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2507_13833_amd import build
        build.build_lib()
    return B.load()


def mat(rows=4, cols=64, stride=None, type_=B.DC_BF16, data=A, reserved=0):
    return B.dc_matrix(data, rows, cols, cols if stride is None else stride, type_, reserved)


def refuses(code, call, *args):
    with pytest.raises(B.DcError) as e:
        call(*args, stream=0)
    assert e.value.code == code


def test_constants_and_structs_match_the_header():
    text = open(os.path.join(ROOT, "include", "dc.h")).read()
    assert re.search(r"#define DC_MAX_HEAD_ROWS\s+\(1 << 22\)", text) and B.DC_MAX_HEAD_ROWS == 1 << 22
    assert C.sizeof(B.dc_norm_params) == 32 and B.dc_norm_params.gate_rows.offset == 24


BAD_MATRICES = [
    (dict(rows=-1), B.DC_ERR_INVALID_ARG), (dict(cols=-1), B.DC_ERR_INVALID_ARG), (dict(stride=63), B.DC_ERR_INVALID_ARG),
    (dict(type_=3), B.DC_ERR_INVALID_ARG), (dict(type_=-1), B.DC_ERR_INVALID_ARG), (dict(reserved=1), B.DC_ERR_INVALID_ARG),
    (dict(data=None), B.DC_ERR_INVALID_ARG), (dict(data=A + 1), B.DC_ERR_INVALID_ARG), (dict(stride=1 << 41), B.DC_ERR_UNSUPPORTED_SIZE),
]


def head(code, hidden=None, weight=None, temperature=1.0, token=A, mask=None, n_top=0, logprob=A, stat=None, entropy=None, top=None,
         top_lp=None, ws=A, ws_bytes=WS):
    refuses(code, B.dc_head_logprob, hidden or mat(), weight or mat(rows=100), temperature, token, mask, n_top, logprob, stat, entropy, top,
            top_lp, ws, ws_bytes, A)


def head_grad(code, hidden=None, weight=None, temperature=1.0, token=A, stat=A, entropy=A, a=A, b=A, gh=True, gw=True, ws=A, ws_bytes=WS):
    gh = mat(data=2 * A) if gh is True else gh
    gw = mat(rows=100, data=3 * A) if gw is True else gw
    refuses(code, B.dc_head_logprob_backward, hidden or mat(), weight or mat(rows=100), temperature, token, None, stat, entropy, a, b, gh, 0, gw,
            ws, ws_bytes, A)


@pytest.mark.parametrize("bad,code", BAD_MATRICES)
def test_head_matrices(bad, code):
    head(code, hidden=mat(**bad))
    head(code, weight=mat(**bad))
    head_grad(code, hidden=mat(**bad))
    head_grad(code, weight=mat(**bad))
    head_grad(code, gh=mat(**bad))
    head_grad(code, gw=mat(**{**dict(rows=100), **bad}))


def test_head():
    for t in (0.0, -1.0, math.nan, math.inf, 1e-40, 1e40):
        head(B.DC_ERR_INVALID_ARG, temperature=t)
    head(B.DC_ERR_INVALID_ARG, hidden=mat(type_=B.DC_F16))                     # types or widths that differ
    head(B.DC_ERR_INVALID_ARG, hidden=mat(cols=65))
    head(B.DC_ERR_INVALID_ARG, hidden=mat(cols=0), weight=mat(rows=100, cols=0))
    head(B.DC_ERR_INVALID_ARG, weight=mat(rows=0))
    head(B.DC_ERR_UNSUPPORTED_SIZE, weight=mat(rows=B.DC_MAX_VOCAB + 1))
    head(B.DC_ERR_UNSUPPORTED_SIZE, hidden=mat(rows=B.DC_MAX_HEAD_ROWS + 1))
    head(B.DC_ERR_UNSUPPORTED_SIZE, hidden=mat(cols=B.DC_MAX_DIM + 1), weight=mat(rows=100, cols=B.DC_MAX_DIM + 1))
    head(B.DC_ERR_INVALID_ARG, token=None)
    head(B.DC_ERR_INVALID_ARG, logprob=None)
    head(B.DC_ERR_INVALID_ARG, token=None, logprob=None)
    head(B.DC_ERR_INVALID_ARG, n_top=-1, top=A)
    head(B.DC_ERR_INVALID_ARG, n_top=2)
    head(B.DC_ERR_INVALID_ARG, weight=mat(rows=4), n_top=5, top=A)
    head(B.DC_ERR_UNSUPPORTED_SIZE, n_top=B.DC_MAX_TOP + 1, top=A)
    for name in ("token", "logprob", "stat", "entropy"):
        head(B.DC_ERR_INVALID_ARG, **{name: A + 2})
    head(B.DC_ERR_INVALID_ARG, n_top=1, top=A + 1)
    for n_top in (0, 5):
        need = B.dc_head_logprob_workspace_bytes(mat(), mat(rows=100), n_top)
        assert need > 0
        head(B.DC_ERR_WORKSPACE, n_top=n_top, top=A, ws_bytes=0)
        head(B.DC_ERR_INVALID_ARG, n_top=n_top, top=A, ws=A + 16)
        head(B.DC_ERR_INVALID_ARG, n_top=n_top, top=A, ws=None)
    assert B.dc_head_logprob_workspace_bytes(mat(), mat(rows=100), B.DC_MAX_TOP + 1) == 0
    assert B.dc_head_logprob_workspace_bytes(mat(cols=65), mat(rows=100), 0) == 0


def test_head_backward():
    bad = B.DC_ERR_INVALID_ARG
    for t in (0.0, math.nan):
        head_grad(bad, temperature=t)
    head_grad(bad, hidden=mat(type_=B.DC_F16))
    head_grad(bad, stat=None)
    head_grad(bad, a=None)
    head_grad(bad, entropy=None)
    for name in ("token", "stat", "entropy", "a", "b"):
        head_grad(bad, **{name: A + 2})
    head_grad(bad, gh=None, gw=None)
    head_grad(bad, gh=mat(rows=5, data=2 * A))
    head_grad(bad, gh=mat(type_=B.DC_F32, data=2 * A))
    head_grad(bad, gw=mat(rows=99, data=2 * A))
    head_grad(bad, gw=mat(rows=100, type_=B.DC_F16, data=2 * A))              # neither the weights' type nor 32 bits
    head_grad(bad, gh=mat())                                                  # in the place of an input
    head_grad(bad, gw=mat(rows=100))
    head_grad(bad, ws=A + 16)
    head_grad(bad, ws=None)
    head_grad(B.DC_ERR_WORKSPACE, ws_bytes=B.dc_head_logprob_backward_workspace_bytes(mat(), mat(rows=100), mat(rows=100)) - 1)
    assert B.dc_head_logprob_backward_workspace_bytes(mat(cols=65), mat(rows=100), None) == 0
    assert B.dc_head_logprob_backward_workspace_bytes(mat(), mat(rows=100), mat(type_=3)) == 0


def test_head_workspaces_grow_with_the_rows():
    for type_ in (B.DC_BF16, B.DC_F32):
        for vocab, dim in ((1, 1), (300, 64), (32000, 1024), (152064, 2048), (152064, 515)):
            w = mat(rows=vocab, cols=dim, type_=type_)
            last = [0, 0, 0]
            for n in [*range(1, 300), 1023, 1024, 1025, 4095, 4096, 8191, 8192, 8193, 65536, 66000, 131072, 262144, 262145, 1 << 21]:
                h = mat(rows=n, cols=dim, type_=type_)
                need = [B.dc_head_logprob_workspace_bytes(h, w, 0), B.dc_head_logprob_workspace_bytes(h, w, min(vocab, 7)),
                        B.dc_head_logprob_backward_workspace_bytes(h, w, mat(rows=vocab, cols=dim, type_=B.DC_F32))]
                assert all(a >= b > 0 or b == 0 for a, b in zip(need, last)), (vocab, dim, n)
                assert need[0] <= need[1]
                last = need


def norm(code, block=None, post=True, gate=None, residual=True, pre=True, prm=None, res_out=True, out=True, stat=A):
    pick = lambda v, d: d if v is True else v  # noqa: E731
    refuses(code, B.dc_residual_norm, block or mat(), pick(post, mat(rows=1)), gate, pick(residual, mat(data=2 * A)), pick(pre, mat(rows=1)),
            prm or B.make_norm(), pick(res_out, mat(data=3 * A)), pick(out, mat(data=4 * A)), stat)


def norm_grad(code, block=None, post=True, gate=None, res_out=True, pre=True, prm=None, stat=A, dh=True, dy=True, gb=True, gr=True,
              g_post=None, g_gate=None, g_pre=None, ws=A, ws_bytes=WS):
    pick = lambda v, d: d if v is True else v  # noqa: E731
    refuses(code, B.dc_residual_norm_backward, block or mat(), pick(post, mat(rows=1)), gate, pick(res_out, mat(data=2 * A)),
            pick(pre, mat(rows=1)), prm or B.make_norm(), stat, pick(dh, mat(data=3 * A)), pick(dy, mat(data=4 * A)), pick(gb, mat(data=5 * A)),
            pick(gr, mat(data=6 * A)), False, g_post, g_gate, g_pre, ws, ws_bytes)


@pytest.mark.parametrize("bad,code", BAD_MATRICES)
def test_norm_matrices(bad, code):
    for name in ("block", "residual", "res_out", "out"):
        norm(code, **{name: mat(**bad)})
    for name in ("post", "gate", "pre"):
        norm(code, **{name: mat(**{**dict(rows=1), **bad})})
    for name in ("block", "res_out", "dh", "dy", "gb", "gr"):
        norm_grad(code, **{name: mat(**bad)})


def test_norm():
    bad = B.DC_ERR_INVALID_ARG
    for eps in (0.0, -1.0, math.nan, math.inf, 1e-50, 1e39):
        norm(bad, prm=B.make_norm(eps))
        norm_grad(bad, prm=B.make_norm(eps))
    for s in (math.nan, math.inf, 1e39):
        norm(bad, prm=B.make_norm(1e-6, s))
        norm(bad, prm=B.make_norm(1e-6, 1.0, s))
    for prm in (B.dc_norm_params(1e-6, 1.0, 1.0, 2, 0), B.dc_norm_params(1e-6, 1.0, 1.0, -1, 0), B.dc_norm_params(1e-6, 1.0, 1.0, 0, 1)):
        norm(bad, prm=prm)
    wide = B.DC_MAX_DIM + 8
    norm(B.DC_ERR_UNSUPPORTED_SIZE, block=mat(cols=wide))
    norm(bad, residual=mat(rows=5, data=2 * A))
    norm(bad, residual=mat(cols=65, data=2 * A))
    norm(bad, res_out=mat(data=3 * A, type_=B.DC_F32))                        # not residual's type
    norm(bad, out=mat(data=4 * A, type_=B.DC_F32))
    norm(bad, post=mat(rows=2))
    norm(bad, pre=mat(rows=1, cols=65))
    norm(bad, pre=None)                                                       # an output without its weight, and the other way round
    norm(bad, out=None)
    norm(bad, gate=mat(rows=4))                                               # rows without gate_rows, and the other way round
    norm(bad, gate=mat(rows=1), prm=B.make_norm(gate_rows=True))
    norm(bad, gate=mat(rows=4, type_=B.DC_F32), prm=B.make_norm(gate_rows=True))
    norm(bad, stat=A + 2)
    norm(bad, res_out=mat(data=2 * A, stride=72))                             # in place with another distance of rows
    norm(bad, out=mat(data=A, stride=72))
    norm(bad, out=mat(data=3 * A))                                            # two outputs in one place, or an output in another input's
    norm(bad, out=mat(data=2 * A))
    norm(bad, res_out=mat(data=A), residual=mat(data=2 * A))


def test_norm_backward():
    bad = B.DC_ERR_INVALID_ARG
    norm_grad(bad, stat=None)
    norm_grad(bad, stat=A + 2)
    norm_grad(bad, dy=None)
    norm_grad(bad, pre=None)
    norm_grad(bad, res_out=None)
    norm_grad(bad, dh=mat(data=3 * A, type_=B.DC_F32))                        # residual_out and its gradient differ in type
    norm_grad(bad, gr=mat(data=6 * A, type_=B.DC_F32))
    norm_grad(bad, dy=mat(data=4 * A, type_=B.DC_F32))
    norm_grad(bad, gb=mat(data=5 * A, type_=B.DC_F32))
    norm_grad(bad, gb=None, gr=None)
    norm_grad(bad, post=None, g_post=mat(rows=1, data=7 * A))
    norm_grad(bad, g_gate=mat(rows=1, data=7 * A))
    norm_grad(bad, pre=None, dy=None, g_pre=mat(rows=1, data=7 * A))
    norm_grad(bad, g_post=mat(rows=2, data=7 * A))
    norm_grad(bad, gate=mat(rows=1, data=8 * A), g_gate=mat(rows=4, data=7 * A))
    norm_grad(bad, gate=mat(data=8 * A), g_gate=mat(data=7 * A, type_=B.DC_F32), prm=B.make_norm(gate_rows=True))
    norm_grad(bad, gb=mat(data=A, stride=72))
    norm_grad(bad, gb=mat(data=4 * A, stride=72))
    norm_grad(bad, gr=mat(data=3 * A, stride=72))
    need = B.dc_residual_norm_backward_workspace_bytes(mat())
    assert need > 0
    norm_grad(B.DC_ERR_WORKSPACE, ws_bytes=need - 1)
    norm_grad(bad, ws=None)
    norm_grad(bad, ws=A + 16)
    assert B.dc_residual_norm_backward_workspace_bytes(mat(cols=B.DC_MAX_DIM + 1)) == 0


def test_norm_workspaces_grow_with_rows_and_columns():
    dims = [1, 64, 512, 513, 2048, 2049, 4096, 8192, 8193, 20000, 65536]
    rows = [1, 2, 255, 256, 257, 1023, 1024, 1025, 100000]
    for d0, d1 in zip(dims, dims[1:]):
        for r0, r1 in zip(rows, rows[1:]):
            big = B.dc_residual_norm_backward_workspace_bytes(mat(rows=r1, cols=d1))
            assert big >= B.dc_residual_norm_backward_workspace_bytes(mat(rows=r0, cols=d1))
            assert big >= B.dc_residual_norm_backward_workspace_bytes(mat(rows=r1, cols=d0))


def test_outputs_in_one_place():
    bad = B.DC_ERR_INVALID_ARG
    head_grad(bad, gh=mat(data=3 * A))                                        # both gradients of the head
    for at in (2, 3, 6):                                                      # residual_out, its gradient, the residual's gradient
        norm_grad(bad, gb=mat(data=at * A))
    for at in (1, 2, 4):                                                      # block, residual_out, grad_out
        norm_grad(bad, gr=mat(data=at * A))
    rows = B.make_norm(gate_rows=True)
    for at in (1, 2, 3, 4, 5, 6, 8):
        norm_grad(bad, gate=mat(data=8 * A), g_gate=mat(data=at * A), prm=rows)
    norm_grad(bad, gate=mat(data=8 * A), gb=mat(data=8 * A), prm=rows)
    norm_grad(bad, gate=mat(data=8 * A), gr=mat(data=8 * A), prm=rows)


def norm_grad_places(**at):
    """A call of every gradient whose arrays lie apart, but for those named: place, and rows' distance or columns where these are given too."""
    spec = dict(block=(4, 1), post=(1, 2), gate=(1, 3), res_out=(4, 4), pre=(1, 5), stat=6, dh=(4, 7), dy=(4, 8), gb=(4, 9), gr=(4, 10),
                g_post=(1, 11), g_gate=(1, 12), g_pre=(1, 13))
    gate_rows = at.pop("gate_rows", False)
    for name in ("gate", "g_gate") if gate_rows else ():
        spec[name] = (4, spec[name][1])
    m = {}
    for name, where in spec.items():
        if name == "stat":
            m[name] = at.get(name, where * A)
            continue
        place = at.get(name, where[1] * A)
        m[name] = mat(rows=where[0], data=place[0], stride=place[1]) if isinstance(place, tuple) else mat(rows=where[0], data=place)
    return [m["block"], m["post"], m["gate"], m["res_out"], m["pre"], B.make_norm(gate_rows=gate_rows), m["stat"], m["dh"], m["dy"], m["gb"],
            m["gr"], False, m["g_post"], m["g_gate"], m["g_pre"], A * 64]


def test_no_output_of_the_norm_in_another_arrays_place():
    """Every output against every other array, but for the places that the contract names: the same place, and a row's end or begin within."""
    accepted = lambda **at: refuses(B.DC_ERR_WORKSPACE, B.dc_residual_norm_backward, *norm_grad_places(**at), 0)  # noqa: E731
    refused = lambda **at: refuses(B.DC_ERR_INVALID_ARG, B.dc_residual_norm_backward, *norm_grad_places(**at), 0)  # noqa: E731
    accepted()
    accepted(gate_rows=True)
    place = dict(block=1, post=2, gate=3, res_out=4, pre=5, stat=6, dh=7, dy=8, gb=9, gr=10, g_post=11, g_gate=12, g_pre=13)
    for out in ("gb", "gr", "g_post", "g_gate", "g_pre"):
        for other, at in place.items():
            if other == out:
                continue
            for rows in (False, True):
                if (out, other) in (("gb", "block"), ("gb", "dy"), ("gr", "dh")):
                    accepted(**{out: at * A}, gate_rows=rows)
                    refused(**{out: (at * A, 72)}, gate_rows=rows)
                    accepted(**{out: (at * A, 72), other: (at * A, 72)}, gate_rows=rows)
                else:
                    refused(**{out: at * A}, gate_rows=rows)
            if other != "stat":
                refused(**{out: at * A + 2})                  # one element further on
                refused(**{out: at * A - 2})
            accepted(**{out: at * A - 4 * 64 * 2 if out in ("gb", "gr") else at * A - 64 * 2})        # ends where the other begins
    # columns of one matrix: rows that interleave, beside each other and one element into each other
    accepted(gb=(9 * A, 128), gr=(9 * A + 128, 128))
    refused(gb=(9 * A, 128), gr=(9 * A + 126, 128))
    refused(gb=(9 * A, 127), gr=(9 * A + 128, 127))
    accepted(gb=(9 * A, 128), g_pre=9 * A + 128, g_post=9 * A + 256 + 128)                            # a row in a gap
    refused(gb=(9 * A, 128), g_pre=9 * A + 130)
    # the forward call
    call = lambda res_out, out, stat: refuses(  # noqa: E731
        B.DC_ERR_INVALID_ARG, B.dc_residual_norm, mat(), mat(rows=1, data=2 * A), mat(rows=1, data=3 * A), mat(data=4 * A), mat(rows=1, data=5 * A),
        B.make_norm(), mat(data=res_out), mat(data=out), stat)
    for at in (1, 2, 3, 5, 7):
        call(at * A, 7 * A, 8 * A)
    for at in (2, 3, 4, 5, 6):
        call(6 * A, at * A, 8 * A)
    for at in (1, 2, 3, 4, 5, 6, 7):
        call(6 * A, 7 * A, at * A)
    call(4 * A + 2, 7 * A, 8 * A)
    call(6 * A, A - 2, 8 * A)
    call(6 * A, 7 * A, 6 * A + 508)                           # statistics at the end of an output


def test_no_gradient_of_the_head_in_another_arrays_place():
    def grad(code, gh, gw):
        refuses(code, B.dc_head_logprob_backward, mat(), mat(rows=100, data=2 * A), 1.0, 3 * A, 4 * A, 5 * A, 6 * A, 7 * A, 8 * A,
                mat(data=gh), 0, mat(rows=100, data=gw), A * 64, 0, A)

    grad(B.DC_ERR_WORKSPACE, 10 * A, 11 * A)
    for at in range(1, 9):                                    # hidden, weight, token, mask, stat, entropy, both gradients
        grad(B.DC_ERR_INVALID_ARG, at * A, 11 * A)
        grad(B.DC_ERR_INVALID_ARG, 10 * A, at * A)
        grad(B.DC_ERR_INVALID_ARG, 10 * A, at * A - 99 * 64 * 2)
    grad(B.DC_ERR_INVALID_ARG, 11 * A + 50 * 128, 11 * A)
    grad(B.DC_ERR_WORKSPACE, 11 * A - 4 * 128, 11 * A)
