"""Refusals of the actor's update: what the entry points and the binding turn down before anything touches a GPU."""
import ctypes as C
import math
import os
import re

import pytest

from paper_2507_13833_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
A = 0x10000                                                   # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module", autouse=True)
def lib():
    if not os.path.exists(B.LIB_PATH):
        from paper_2507_13833_amd import build
        build.build_lib()
    return B.load()


def mat(rows=4, cols=100, stride=None, type_=B.DC_BF16, data=A, reserved=0):
    return B.dc_matrix(data, rows, cols, cols if stride is None else stride, type_, reserved)


def refuses(code, call, *args):
    with pytest.raises(B.DcError) as e:
        call(*args, stream=0)
    assert e.value.code == code


def test_constants_and_structs_match_the_header():
    text = open(os.path.join(ROOT, "include", "dc.h")).read()
    for name in ("DC_MAX_TOP", "DC_MAX_TENSORS", "DC_STATE_BLOCK"):
        assert re.search(rf"#define\s+{name}\s+{getattr(B, name)}\b", text)
    assert "#define DC_MAX_VOCAB      (1 << 24)" in text and B.DC_MAX_VOCAB == 1 << 24
    assert "#define DC_NO_TOKEN       (-1)" in text and B.DC_NO_TOKEN == -1
    for name, val in re.findall(r"\b(DC_(?:F32|BF16|F16|E4M3)) = (\d)", text):
        assert getattr(B, name) == int(val)
    assert C.sizeof(B.dc_matrix) == 40 and C.sizeof(B.dc_adamw_tensor) == 88 and C.sizeof(B.dc_adamw_params) == 40
    assert B.dc_adamw_tensor.n.offset == 56 and B.dc_adamw_tensor.param_type.offset == 72
    assert "vocabulary" in B.strerror(B.DC_ERR_TOKEN_RANGE)


BAD_MATRICES = [
    (dict(rows=-1), B.DC_ERR_INVALID_ARG), (dict(cols=-1), B.DC_ERR_INVALID_ARG), (dict(stride=99), B.DC_ERR_INVALID_ARG),
    (dict(type_=3), B.DC_ERR_INVALID_ARG), (dict(type_=-1), B.DC_ERR_INVALID_ARG), (dict(reserved=1), B.DC_ERR_INVALID_ARG),
    (dict(data=None), B.DC_ERR_INVALID_ARG), (dict(data=A + 1), B.DC_ERR_INVALID_ARG),
    (dict(data=A + 2, type_=B.DC_F32), B.DC_ERR_INVALID_ARG),
    (dict(rows=1 << 30, stride=1 << 31), B.DC_ERR_UNSUPPORTED_SIZE), (dict(stride=1 << 41), B.DC_ERR_UNSUPPORTED_SIZE),
]


@pytest.mark.parametrize("bad,code", BAD_MATRICES)
def test_matrices(bad, code):
    good = mat(**{k: v for k, v in bad.items() if k in ("rows", "cols")}) if not {"rows", "cols"} & set(bad) else mat()
    refuses(code, B.dc_token_logprob, mat(**bad), 1.0, A, None, 0, A, None, None, None, None, None, 0, A)
    refuses(code, B.dc_token_logprob_backward, mat(**bad), 1.0, A, None, A, None, A, None, mat(**bad), A)
    refuses(code, B.dc_token_logprob_backward, good, 1.0, A, None, A, None, A, None, mat(**bad), A)
    refuses(code, B.dc_embedding, mat(**bad), A, 1.0, good, A)
    refuses(code, B.dc_embedding, good, A, 1.0, mat(**bad), A)
    refuses(code, B.dc_embedding_backward, mat(**bad), A, 1.0, 0, good, A, 1 << 40, A)
    refuses(code, B.dc_embedding_backward, good, A, 1.0, 0, mat(**bad), A, 1 << 40, A)


def test_logprob():
    def call(code, x=None, temperature=1.0, token=A, mask=None, n_top=0, out=A, stat=None, entropy=None, top=None, top_lp=None,
             ws=None, ws_bytes=0):
        refuses(code, B.dc_token_logprob, x or mat(), temperature, token, mask, n_top, out, stat, entropy, top, top_lp, ws,
                ws_bytes, A)
    for t in (0.0, -1.0, math.nan, math.inf, 1e-40, 1e40):
        call(B.DC_ERR_INVALID_ARG, temperature=t)
    call(B.DC_ERR_INVALID_ARG, x=mat(cols=0))
    call(B.DC_ERR_UNSUPPORTED_SIZE, x=mat(cols=B.DC_MAX_VOCAB + 1))
    call(B.DC_ERR_INVALID_ARG, token=None)                    # a result without its token, and the other way round
    call(B.DC_ERR_INVALID_ARG, out=None)
    call(B.DC_ERR_INVALID_ARG, token=None, out=None)          # nothing asked for
    call(B.DC_ERR_INVALID_ARG, n_top=-1, top=A)
    call(B.DC_ERR_INVALID_ARG, n_top=2)                       # alternatives without a place to put them
    call(B.DC_ERR_INVALID_ARG, x=mat(cols=4), n_top=5, top=A)
    call(B.DC_ERR_UNSUPPORTED_SIZE, n_top=B.DC_MAX_TOP + 1, top=A)
    for name in ("token", "out", "stat", "entropy"):
        call(B.DC_ERR_INVALID_ARG, **{name: A + 2})
    call(B.DC_ERR_INVALID_ARG, n_top=1, top=A + 1)
    call(B.DC_ERR_INVALID_ARG, n_top=1, top=A, top_lp=A + 1)
    large = mat(rows=2, cols=152064)
    need = B.dc_token_logprob_workspace_bytes(large, 5)
    if need:
        call(B.DC_ERR_WORKSPACE, x=large, n_top=5, top=A, ws=A, ws_bytes=need - 1)
        call(B.DC_ERR_INVALID_ARG, x=large, n_top=5, top=A, ws=A + 16, ws_bytes=need)
        call(B.DC_ERR_INVALID_ARG, x=large, n_top=5, top=A, ws=None, ws_bytes=need)
    assert B.dc_token_logprob_workspace_bytes(mat(rows=-1), 5) == 0
    assert B.dc_token_logprob_workspace_bytes(large, B.DC_MAX_TOP + 1) == 0


def test_logprob_backward():
    def call(x=None, g=None, token=A, stat=A, entropy=A, gl=A, ge=A, temperature=1.0):
        refuses(B.DC_ERR_INVALID_ARG, B.dc_token_logprob_backward, x or mat(), temperature, token, None, stat, entropy, gl, ge,
                g or mat(data=2 * A), A)
    call(temperature=0.0)
    call(g=mat(data=2 * A, rows=3))
    call(g=mat(data=2 * A, cols=99))
    call(g=mat(data=2 * A, type_=B.DC_F16))
    call(g=mat(stride=101))                                   # in place, but not the same rows
    call(stat=None)
    call(gl=None)
    call(entropy=None)                                        # the entropy's gradient without the entropy
    for name in ("token", "stat", "entropy", "gl", "ge"):
        call(**{name: A + 2})


def test_embedding():
    w, out = mat(rows=50, cols=64), mat(rows=9, cols=64, data=2 * A)
    bad = B.DC_ERR_INVALID_ARG
    refuses(bad, B.dc_embedding, w, None, 1.0, out, A)
    refuses(bad, B.dc_embedding, w, A + 2, 1.0, out, A)
    refuses(bad, B.dc_embedding, w, A, 1.0, mat(rows=9, cols=65), A)
    for s in (math.nan, math.inf, 1e39):
        refuses(bad, B.dc_embedding, w, A, s, out, A)
        refuses(bad, B.dc_embedding_backward, out, A, s, 0, w, A, 1 << 40, A)
    refuses(B.DC_ERR_UNSUPPORTED_SIZE, B.dc_embedding, mat(rows=B.DC_MAX_VOCAB + 1, cols=64), A, 1.0, out, A)
    refuses(bad, B.dc_embedding_backward, out, None, 1.0, 0, w, A, 1 << 40, A)
    refuses(bad, B.dc_embedding_backward, out, A + 1, 1.0, 0, w, A, 1 << 40, A)
    refuses(bad, B.dc_embedding_backward, mat(rows=9, cols=65), A, 1.0, 0, w, A, 1 << 40, A)
    refuses(B.DC_ERR_UNSUPPORTED_SIZE, B.dc_embedding_backward, mat(rows=(1 << 24) + 1, cols=64), A, 1.0, 0, w, A, 1 << 40, A)
    refuses(B.DC_ERR_UNSUPPORTED_SIZE, B.dc_embedding_backward, out, A, 1.0, 0, mat(rows=B.DC_MAX_VOCAB + 1, cols=64), A, 1 << 40, A)
    need = B.dc_embedding_backward_workspace_bytes(out, w)
    if need:
        refuses(B.DC_ERR_WORKSPACE, B.dc_embedding_backward, out, A, 1.0, 0, w, A, need - 1, A)
        refuses(bad, B.dc_embedding_backward, out, A, 1.0, 0, w, A + 128, need, A)
        refuses(bad, B.dc_embedding_backward, out, A, 1.0, 0, w, None, need, A)


class Tensors:
    """What AdamwTensors holds, made of addresses."""

    def __init__(self, *items):
        self.array = (B.dc_adamw_tensor * max(1, len(items)))(*items)
        self.n = len(items)


def tensor(n=1000, param_type=B.DC_BF16, grad_type=B.DC_BF16, state_type=B.DC_E4M3, param=A, master=A, grad=A, m=A, v=A, ms=A, vs=A,
           decay=0.1, reserved=0):
    return B.dc_adamw_tensor(param, master, grad, m, v, ms, vs, n, decay, param_type, grad_type, state_type, reserved)


BAD_TENSORS = [
    (dict(n=-1), B.DC_ERR_INVALID_ARG), (dict(param_type=B.DC_E4M3), B.DC_ERR_INVALID_ARG), (dict(grad_type=7), B.DC_ERR_INVALID_ARG),
    (dict(state_type=B.DC_BF16), B.DC_ERR_INVALID_ARG), (dict(param=None), B.DC_ERR_INVALID_ARG), (dict(grad=None), B.DC_ERR_INVALID_ARG),
    (dict(m=None), B.DC_ERR_INVALID_ARG), (dict(v=None), B.DC_ERR_INVALID_ARG), (dict(ms=None), B.DC_ERR_INVALID_ARG),
    (dict(vs=None), B.DC_ERR_INVALID_ARG), (dict(param=A + 1), B.DC_ERR_INVALID_ARG), (dict(master=A + 2), B.DC_ERR_INVALID_ARG),
    (dict(m=A + 2, state_type=B.DC_F32), B.DC_ERR_INVALID_ARG), (dict(ms=A + 1), B.DC_ERR_INVALID_ARG),
    (dict(decay=-0.1), B.DC_ERR_INVALID_ARG), (dict(decay=math.nan), B.DC_ERR_INVALID_ARG), (dict(reserved=1), B.DC_ERR_INVALID_ARG),
    (dict(n=(1 << 40) + 1), B.DC_ERR_UNSUPPORTED_SIZE),
]


@pytest.mark.parametrize("bad,code", BAD_TENSORS)
def test_adamw_tensors(bad, code):
    t = Tensors(tensor(), tensor(**bad))
    assert B.dc_adamw_table_bytes(t) == 0
    refuses(code, B.dc_adamw_table, t, A, 1 << 40)
    refuses(code, B.dc_adamw, t, B.make_adamw(1e-3), None, A, 1 << 40, A)


def test_adamw():
    t = Tensors(tensor(), tensor(n=5000, state_type=B.DC_F32, ms=None, vs=None, master=None))
    need = B.dc_adamw_table_bytes(t)
    assert need > 0 and need % 256 == 0
    refuses(B.DC_ERR_WORKSPACE, B.dc_adamw_table, t, A, need - 1)
    refuses(B.DC_ERR_WORKSPACE, B.dc_adamw, t, B.make_adamw(1e-3), None, A, need - 1, A)
    refuses(B.DC_ERR_INVALID_ARG, B.dc_adamw_table, t, None, need)
    refuses(B.DC_ERR_INVALID_ARG, B.dc_adamw_table, t, A + 8, need)
    refuses(B.DC_ERR_INVALID_ARG, B.dc_adamw, t, B.make_adamw(1e-3), A + 2, A, need, A)
    for kw in (dict(lr=-1.0), dict(lr=math.nan), dict(lr=math.inf), dict(lr=1e-3, beta1=1.0), dict(lr=1e-3, beta1=-0.1),
               dict(lr=1e-3, beta2=1.0), dict(lr=1e-3, beta2=math.nan), dict(lr=1e-3, eps=0.0), dict(lr=1e-3, eps=1e-60),
               dict(lr=1e-3, eps=math.inf), dict(lr=1e-3, step=0)):
        refuses(B.DC_ERR_INVALID_ARG, B.dc_adamw, t, B.make_adamw(**kw), None, A, need, A)


class FakeTensor:
    """As much of a device tensor as the binding looks at."""

    def __init__(self, shape, dtype="torch.float32", stride=None, cuda=True):
        import torch
        self.shape, self.is_cuda = torch.Size(shape), cuda
        self.dtype = getattr(torch, dtype.split(".")[1])
        self._stride = stride or tuple(math.prod(shape[i + 1:]) for i in range(len(shape)))

    def dim(self): return len(self.shape)
    def stride(self, i=None): return self._stride if i is None else self._stride[i]
    def numel(self): return math.prod(self.shape)
    def data_ptr(self): return A
    def is_contiguous(self): return True


def test_binding_checks_tensors():
    for t in (FakeTensor((4, 100), cuda=False), FakeTensor((100,)), FakeTensor((4, 100), stride=(1, 4)),
              FakeTensor((4, 100), stride=(50, 1)), FakeTensor((4, 100), dtype="torch.int32")):
        with pytest.raises(TypeError):
            B.make_matrix(t)
    m = B.make_matrix(FakeTensor((4, 100), dtype="torch.float16", stride=(131, 1)))
    assert (m.n_rows, m.n_cols, m.row_stride, m.type) == (4, 100, 131, B.DC_F16)
    logits = mat()
    with pytest.raises(TypeError):                            # 64-bit ids
        B.dc_token_logprob(logits, 1.0, FakeTensor((4,), "torch.int64"), None, 0, FakeTensor((4,)), None, None, None, None, None,
                           0, A, stream=0)
    with pytest.raises(ValueError):                           # too few
        B.dc_token_logprob(logits, 1.0, FakeTensor((3,), "torch.int32"), None, 0, FakeTensor((4,)), None, None, None, None, None,
                           0, A, stream=0)
    with pytest.raises(ValueError):
        B.dc_embedding(mat(rows=50), FakeTensor((3,), "torch.int32"), 1.0, mat(), A, stream=0)
    with pytest.raises(ValueError):
        B.AdamwTensors([dict(param=FakeTensor((8,)), grad=FakeTensor((7,)), exp_avg=FakeTensor((8,)), exp_avg_sq=FakeTensor((8,)))])
    with pytest.raises(TypeError):
        B.AdamwTensors([dict(param=FakeTensor((8,)), grad=FakeTensor((8,)), exp_avg=FakeTensor((8,)),
                             exp_avg_sq=FakeTensor((8,), "torch.float8_e4m3fn"))])


def test_workspaces_and_limits():
    """Sizes whose rows are cut into parts need a workspace; limits of the embedding."""
    big = mat(rows=2, cols=152064, type_=B.DC_F32)
    for n_top in (0, 5):
        need = B.dc_token_logprob_workspace_bytes(big, n_top)
        assert need > 0
        args = (big, 1.0, A, None, n_top, A, None, None, A if n_top else None, None)
        refuses(B.DC_ERR_WORKSPACE, B.dc_token_logprob, *args, A, need - 1, A)
        refuses(B.DC_ERR_INVALID_ARG, B.dc_token_logprob, *args, A + 16, need, A)
        refuses(B.DC_ERR_INVALID_ARG, B.dc_token_logprob, *args, None, need, A)
    wide = mat(rows=9, cols=B.DC_MAX_DIM + 8)
    refuses(B.DC_ERR_UNSUPPORTED_SIZE, B.dc_embedding, wide, A, 1.0, wide, A)
    refuses(B.DC_ERR_UNSUPPORTED_SIZE, B.dc_embedding_backward, wide, A, 1.0, 0, wide, A, 1 << 40, A)
    many = mat(rows=1 << 24, cols=32768)
    refuses(B.DC_ERR_UNSUPPORTED_SIZE, B.dc_embedding_backward, many, A, 1.0, 0, mat(rows=9, cols=32768), A, 1 << 62, A)
    assert B.dc_embedding_backward_workspace_bytes(wide, wide) == 0
    assert B.dc_embedding_backward_workspace_bytes(mat(rows=0, cols=8), mat(rows=9, cols=8)) > 0


def test_nothing_to_do_is_no_error():
    """Calls without rows return before anything is enqueued, whatever their other pointers."""
    none = mat(rows=0, data=None)
    B.dc_token_logprob(none, 1.0, None, None, 3, None, None, None, None, None, None, 0, None, stream=0)
    B.dc_token_logprob_backward(none, 1.0, None, None, None, None, None, None, none, None, stream=0)
    B.dc_embedding(mat(rows=50), None, 1.0, none, None, stream=0)
    t = Tensors()
    need = B.dc_adamw_table_bytes(t)
    B.dc_adamw_table(t, A, need, stream=0)
    B.dc_adamw(t, B.make_adamw(1e-3), None, A, need, None, stream=0)


def test_adamw_eps_that_32_bits_cannot_divide_by():
    t = Tensors(tensor())
    need = B.dc_adamw_table_bytes(t)
    for eps in (1e-39, 1e-31, 1e31, 1e38):                    # a denormal; what has no normal reciprocal
        refuses(B.DC_ERR_INVALID_ARG, B.dc_adamw, t, B.make_adamw(1e-3, eps=eps), None, A, need, A)


def test_adamw_tensors_outlive_the_dicts_they_came_in():
    """The array holds addresses, so what they belong to stays, also when a program puts another gradient, or none, in its dict."""
    import gc
    import weakref
    item = {k: FakeTensor((8,)) for k in ("param", "grad", "exp_avg", "exp_avg_sq")}
    seen = {k: weakref.ref(t) for k, t in item.items()}
    items = [item]
    t = B.AdamwTensors(items)
    item["grad"] = None
    item["param"] = FakeTensor((8,))
    items.clear()
    del item
    gc.collect()
    assert t.n == 1 and all(ref() is not None for ref in seen.values())
    del t
    gc.collect()
    assert all(ref() is None for ref in seen.values())


def test_embedding_backward_workspace_of_the_largest_call_serves_smaller_ones():
    """A program that sizes it once, for its largest micro-batch: the sizes do not fall where the kernels are cut otherwise."""
    def size(tokens, dim):
        return B.dc_embedding_backward_workspace_bytes(mat(rows=tokens, cols=dim), mat(rows=50000, cols=dim))
    counts = sorted({n + d for k in (0, 16, 32, 512, 1024, 8192, 16384, 1 << 24) for n in (k, 131072 // max(1, k // 512)) for d in (-1, 0, 1)
                     if 0 <= n + d <= 1 << 24} | {21845, 26214, 32767, 32768, 40000, 43690, 43691, 65535, 65536, 87381, 131071, 131072, 262144})
    dims = [1, 100, 511, 512, 513, 1024, 1025, 1536, 2047, 2048, 2049, 4096, 8192, 16384, 16385, 65536]
    of = {(n, d): size(n, d) for n in counts for d in dims if n * d <= 1 << 38}
    assert all(v > 0 and v % 256 == 0 for k, v in of.items() if k[0] > 0)
    for n, d in of:
        for n2, d2 in ((counts[min(counts.index(n) + 1, len(counts) - 1)], d), (n, dims[min(dims.index(d) + 1, len(dims) - 1)])):
            if (n2, d2) in of:
                assert of[n, d] <= of[n2, d2], (n, d, n2, d2)
    for tokens, dim in ((32767, 2048), (16700, 2048), (40000, 2048), (65535, 1024), (131071, 512), (9000, 2048)):
        # refused for less than the call needs, whatever the largest call would need: half its pieces are too few
        refuses(B.DC_ERR_WORKSPACE, B.dc_embedding_backward, mat(rows=tokens, cols=dim), A, 1.0, 0, mat(rows=50000, cols=dim), A,
                size(tokens, dim) // 2, A)


def test_logprob_workspace_of_the_largest_call_serves_smaller_ones():
    """A program that sizes it once, for its largest batch, decodes with fewer rows: the size does not fall with them."""
    for cols in (1, 32000, 32769, 65537, 70000, 131073, 152064, 1 << 20, B.DC_MAX_VOCAB):
        for type_ in (B.DC_F32, B.DC_BF16, B.DC_F16):
            for n_top in (0, 1, 5, 20, 64):
                if n_top > cols:
                    continue
                size = [B.dc_token_logprob_workspace_bytes(mat(rows=r, cols=cols, type_=type_), n_top) for r in (*range(131), 256, 257, 1 << 20)]
                assert all(a <= b for a, b in zip(size, size[1:])), (cols, type_, n_top)
                assert n_top == 0 or size[64] >= B.dc_token_logprob_workspace_bytes(mat(rows=64, cols=cols, type_=type_), n_top - 1)
    assert B.dc_token_logprob_workspace_bytes(mat(rows=100, cols=152064), 5) > 0


def test_adamw_factors_that_32_bits_do_not_hold():
    t, strong = Tensors(tensor()), Tensors(tensor(decay=0.1), tensor(n=0, decay=0.0), tensor(decay=1e10))
    need = max(B.dc_adamw_table_bytes(t), B.dc_adamw_table_bytes(strong))
    for kw in (dict(lr=1e39), dict(lr=3e38, beta1=0.9), dict(lr=1e308), dict(lr=1e30, beta1=1 - 1e-12)):
        refuses(B.DC_ERR_INVALID_ARG, B.dc_adamw, t, B.make_adamw(**kw), None, A, need, A)
    refuses(B.DC_ERR_INVALID_ARG, B.dc_adamw, strong, B.make_adamw(1e30), None, A, need, A)
    refuses(B.DC_ERR_INVALID_ARG, B.dc_adamw, strong, B.make_adamw(1e300, step=1 << 40), None, A, need, A)
