"""The operators at a token model's two ends at the limits of their arguments, as far as no device is needed."""
import ctypes as C
import random

import pytest
import torch

from paper_2609_29505_gb300 import binding

OK, ARG = binding.SGD_OK, binding.SGD_ERR_ARG
P = 1 << 20  # an address that nothing reads


@pytest.fixture(scope="module")
def lib():
    from paper_2609_29505_gb300 import build
    build.build()
    return binding.lib()


@pytest.mark.parametrize("rows,d", [(1, 4), (64, 64), (65, 1152), (5000, 4096), ((1 << 27) - 1, 4)])
def test_norm_grad_workspace_of_one_sample(lib, rows, d):
    """Every period that holds all rows means one sample, up to the largest integer."""
    n = C.c_int64(0)
    assert lib.sgd_kernel_norm_grad_workspace(rows, d, rows, C.byref(n)) == OK
    want = n.value
    assert want > 0
    for per in (rows + 1, 2 ** 31 - 1, 2 ** 31 - 48, 2 ** 31 - rows, 2 ** 31 - rows + 1):
        assert lib.sgd_kernel_norm_grad_workspace(rows, d, min(per, 2 ** 31 - 1), C.byref(n)) == OK
        assert n.value == want, per
    for per in (2 ** 31, 2 ** 32 + 1, 2 ** 40):
        assert binding.sgd_kernel_norm_grad_workspace(rows, d, per) == want


@pytest.mark.parametrize("handle,want", [(0, "default"), (7, "external 7"), ("an object", "an object")])
def test_workspace_of_a_call_belongs_to_its_stream(monkeypatch, handle, want):
    """torch's allocator gives memory to the next user of the stream that it was allocated on: that has to be the call's."""
    import contextlib
    on, got = [], []
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda h, device=None: f"external {h}" if h else "a stream of the pool")
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: "default")
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())

    @contextlib.contextmanager
    def stream(s):
        on.append(s)
        yield
        on.pop()
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch, "empty", lambda n, **kw: got.append((n, on[-1])))
    assert binding._workspace(None, 64, torch.device("cuda:0"), handle)[1] == 64
    assert got == [(64, want)]


class _Shape:
    """What the checks see of a tensor on a device, without its memory."""
    is_cuda, device, dtype = True, torch.device("cuda:0"), torch.float16

    def __init__(self, *shape, dtype=torch.float16):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (self.shape[1], 1)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        raise AssertionError("the address is not asked for")


def test_sizes_of_more_than_32_bits_are_refused():
    """The library's sizes are 32 bits: a table of 2^32 + 3 rows would be one of 3."""
    many, wide, few = _Shape(2 ** 32 + 3, 1), _Shape(2, 2 ** 32 + 3), _Shape(4, 1)
    ids = _Shape(4, dtype=torch.int32)
    for call in (lambda: binding.sgd_kernel_sample(many, None, None), lambda: binding.sgd_kernel_sample(wide, None, None),
                 lambda: binding.sgd_kernel_logprobs(many), lambda: binding.sgd_kernel_embedding(many, ids, few),
                 lambda: binding.sgd_kernel_embedding(few, ids, many), lambda: binding.sgd_kernel_embedding_grad(few, ids, many),
                 lambda: binding.sgd_kernel_embedding_grad(many, ids, few), lambda: binding.sgd_kernel_norm_grad(many, many, 0, dh=many),
                 lambda: binding.sgd_kernel_norm_grad(few, wide, 0), lambda: binding.sgd_kernel_embedding_grad_workspace(2 ** 32 + 1, 8, 8),
                 lambda: binding.sgd_kernel_embedding_grad_workspace(1, 2 ** 31, 8), lambda: binding.sgd_kernel_embedding_grad_workspace(1, 8, 2 ** 33),
                 lambda: binding.sgd_kernel_norm_grad_workspace(2 ** 32 + 1, 8), lambda: binding.sgd_kernel_norm_grad_workspace(1, 2 ** 32 + 8)):
        with pytest.raises(ValueError, match="32-bit"):
            call()


def _sample(lib, **kw):
    a = dict(logits=P, dtype=0, ld=64, rows=8, vocab=60, scale=1.0, top_k=0, top_p=1.0, min_p=0.0, uniforms=2 * P, row_ids=3 * P, row_id=0,
             ids=4 * P, logprobs=5 * P, stream=None)
    a.update(kw)
    return lib.sgd_kernel_sample(*a.values())


@pytest.mark.parametrize("name", ["ids", "logprobs"])
@pytest.mark.parametrize("at", [P, P + 4, P + 7 * 128 + 116, 2 * P, 2 * P + 60, 3 * P, 3 * P - 28, 3 * P + 28, P + 7 * 128 - 4])
def test_sample_refuses_overlaps(lib, name, at):
    assert _sample(lib, **{name: at}) == ARG and b"overlaps" in lib.sgd_last_error()


def test_sample_refuses_outputs_that_overlap(lib):
    for at in (4 * P, 4 * P + 28, 4 * P - 28):
        assert _sample(lib, logprobs=at) == ARG and b"overlaps" in lib.sgd_last_error()


def _norm_grad(lib, **kw):
    a = dict(h=P, dout=2 * P, dtype=1, rows=6, d=8, kind=1, g=3 * P, b=4 * P, scale=5 * P, ld_mod=16, rows_per_batch=2, eps=1e-6,
             residual=6 * P, dh=7 * P, dg=8 * P, db=9 * P, dshift=10 * P, dscale=11 * P, ld_dmod=16, workspace=12 * P, workspace_bytes=1 << 16,
             stream=None)
    a.update(kw)
    return lib.sgd_kernel_norm_grad(*a.values())


@pytest.mark.parametrize("name,at", [
    ("dg", P), ("dg", P + 176), ("dg", 2 * P + 80), ("dg", 3 * P), ("db", 4 * P - 16), ("dg", 5 * P), ("dg", 6 * P), ("dg", 7 * P + 176), ("db", 8 * P + 16),
    ("dshift", P), ("dshift", 5 * P), ("dshift", 5 * P + 28), ("dshift", 7 * P), ("dshift", 8 * P), ("dscale", 10 * P), ("dscale", 10 * P + 28),
    ("dscale", 10 * P - 28), ("dscale", 3 * P), ("dh", 3 * P), ("dh", 5 * P), ("dh", 4 * P), ("dh", 8 * P - 32),
    ("workspace", P), ("workspace", 2 * P), ("workspace", 3 * P), ("workspace", 5 * P + 128), ("workspace", 6 * P), ("workspace", 7 * P),
    ("workspace", 8 * P), ("workspace", 10 * P + 64), ("workspace", 11 * P),
])
def test_norm_grad_refuses_overlaps(lib, name, at):
    assert _norm_grad(lib, **{name: at}) == ARG and b"overlap" in lib.sgd_last_error()


def test_overlaps_of_matrices(lib):
    """dshift and scale as parts of one memory: refused where they have a byte in common, and where their strides differ and their
    extents meet.  (Without a workspace: what is not refused for the overlap is for that, and nothing is launched.)"""
    rng = random.Random(3)
    seen = {True: 0, False: 0}
    for _ in range(3000):
        rows, d = rng.randint(1, 7), 4 * rng.randint(1, 4)
        per = rng.randint(1, 3)
        samples = -(-rows // per)
        ld = d + rng.choice([0, 1, 3, d, 2 * d])
        ld2 = ld if rng.random() < 0.7 else d + rng.choice([0, 2, d])
        at = 5 * P + 4 * rng.randint(-samples * ld - 3, samples * ld + 3)
        a = {5 * P + 4 * (i * ld + j) for i in range(samples) for j in range(d)}
        b = {at + 4 * (i * ld2 + j) for i in range(samples) for j in range(d)}
        want = bool(a & b)
        if ld != ld2 and ld != d and ld2 != d and samples > 1:
            want = max(min(a), min(b)) <= min(max(a), max(b))
        got = _norm_grad(lib, rows=rows, d=d, rows_per_batch=per, ld_mod=ld, ld_dmod=ld2, dshift=at, dscale=None, workspace=None)
        assert got == ARG
        assert (b"overlaps" in lib.sgd_last_error()) == want, (rows, d, per, ld, ld2, at)
        assert want or b"workspace" in lib.sgd_last_error()
        seen[want] += 1
    assert min(seen.values()) > 300


def _embedding(lib, **kw):
    a = dict(table=P, dtype=1, ld=8, vocab=4, d=8, ids=P << 8, rows=2, scale=1.0, out=(P << 8) + 4, out_dtype=2, ld_out=8, stream=None)
    a.update(kw)
    return lib.sgd_kernel_embedding(*a.values())


def test_overlaps_of_the_largest_matrices(lib):
    """Extents that pass 64 bits: of 2^31 - 1 rows, 2^40 fp32 values apart."""
    huge = dict(table=P, dtype=2, ld=1 << 40, vocab=2 ** 31 - 1, d=8, ids=P >> 1)
    for row in (1, 3, 1 << 20):
        assert _embedding(lib, **huge, rows=1, out=P + (row << 42) + 16) == ARG and b"overlaps" in lib.sgd_last_error()


@pytest.mark.parametrize("rows,d,chunk", [(1, 1, 8), (17, 300, 8), (1000, 4096, 8), (4000, 1024, 8), (4103, 4096, 8), (4104, 4096, 16), (8207, 4096, 16),
                                          (8208, 4096, 32), (16391, 1024, 8), (16392, 1024, 16), (32783, 64, 16), (32784, 64, 32), (65537, 1024, 32),
                                          (1 << 20, 64, 32), (6144, 64, 8), (6145, 64, 8)])
def test_embedding_grad_workspace(lib, rows, d, chunk):
    """Tokens and order, twice above the 6144 rows that are sorted by counting, with 1 KB of counts per 1024 rows there; two rows of partial sums
    per chunk of 8, 16 or 32 rows: the largest that leaves 2048 pieces of 1024 columns, or 8."""
    n = C.c_int64(0)
    assert lib.sgd_kernel_embedding_grad_workspace(rows, 1000, d, C.byref(n)) == OK
    sums = 8 * -(-rows // chunk) * (-(-d // 8) * 8)
    sort = 8 * rows if rows <= 6144 else 16 * rows
    assert sums + sort <= n.value <= sums + sort + (0 if rows <= 6144 else rows + 1024) + 6 * 256
