"""Host side of scored attention and dropout, without a GPU: the refusals of the
C ABI, the workspace sizes, the bucket map, and the reference generator."""
import ctypes as C

import numpy as np
import pytest

from paper_2504_13850_gb300 import api, build


@pytest.fixture(scope="module", autouse=True)
def lib():
    build.build()


def spec(**over):
    f = dict(batch=2, len=200, heads=4, kv_heads=2, head_dim=64, dtype=api.DTYPE_BF16, causal=1, buckets=0, reach=0,
             scale=0.125, softcap=0.0)
    f.update(over)
    s = api.fo_attention_spec()
    for n, v in f.items():
        setattr(s, n, v)
    return s


def workspace(s, backward=0):
    return api.lib().fo_attention_workspace(C.byref(s), backward)


def test_workspace_sizes():
    assert workspace(spec()) == 0
    rows = 2 * 4 * 256
    assert workspace(spec(), 1) == 2 * rows * 4                       # lse and D, padded to 128 tokens
    assert workspace(spec(documents=256)) == 2 * 256 * 4 + 256
    assert workspace(spec(len=0)) == 0 and workspace(spec(batch=0), 1) == 0


@pytest.mark.parametrize("over,what", [
    ({"batch": -1}, "batch"), ({"len": -1}, "len"), ({"len": (1 << 20) + 1}, "len"), ({"heads": 0}, "heads"),
    ({"kv_heads": 3}, "multiple"), ({"kv_heads": 0}, "multiple"), ({"head_dim": 0}, "head_dim"),
    ({"head_dim": 129}, "head_dim"), ({"dtype": 2}, "dtype"), ({"scale": 0.0}, "scale"),
    ({"scale": float("inf")}, "scale"), ({"softcap": -1.0}, "softcap"), ({"softcap": float("nan")}, "softcap"),
    ({"causal": 0, "prefix": 256}, "prefix"), ({"table": 256, "slopes": 256}, "one of"),
    ({"table": 256}, "buckets"), ({"table": 256, "buckets": 129, "reach": 4}, "buckets"),
    ({"len": 1 << 20, "batch": 1 << 20}, "tiles")])
def test_bad_specs_are_refused(over, what):
    s = spec(**over)
    assert workspace(s) == -1 and what in api.last_error()
    assert api.lib().fo_attention_forward(C.byref(s), *[None] * 4, None, None, 0, None) == api.ERR_ARG
    assert api.lib().fo_attention_backward(C.byref(s), *[None] * 5, None, *[None] * 3, None, None, 0, None) == api.ERR_ARG


def test_bad_bucket_maps_are_refused():
    m = np.zeros(2 * 16 + 1, np.uint8)
    ok = dict(table=256, buckets=8, reach=16, bucket_of_host=m.ctypes.data)
    assert workspace(spec(**ok)) == 0
    for reach in (0, 513):
        assert workspace(spec(**dict(ok, reach=reach))) == -1 and "reach" in api.last_error()
    m[5] = 8
    assert workspace(spec(**ok)) == -1 and "entry 5" in api.last_error()


def test_bad_tensors_and_workspaces_are_refused():
    L = api.lib()
    s = spec(documents=256)

    def t(p=4096, b=200 * 256, l=256, h=64):
        return C.byref(api.fo_strided(p, b, l, h))

    def forward(q=t(), o=t(), lse=4096, ws=4096, n=1 << 20):
        return L.fo_attention_forward(C.byref(s), q, t(), t(), o, lse, ws, n, None)

    for kw, what in (({"q": None}, "null q"), ({"q": t(p=0)}, "null q"), ({"q": t(p=4097)}, "misaligned q"),
                     ({"q": t(l=-1)}, "strides of q"), ({"o": t(l=0)}, "strides of o"),
                     ({"o": t(l=255)}, "strides of o"), ({"o": t(b=200 * 256 - 1)}, "strides of o"),
                     ({"o": t(h=63)}, "strides of o"), ({"lse": None}, "lse"),
                     ({"ws": None}, "workspace"), ({"ws": 4100}, "workspace"), ({"n": 100}, "needed")):
        assert forward(**kw) == api.ERR_ARG and what in api.last_error(), kw
    bare = spec()
    rc = L.fo_attention_backward(C.byref(bare), *[t()] * 4, 4096, *[t()] * 4, 4096, 4096, 1 << 20, None)
    assert rc == api.ERR_ARG and "dtable" in api.last_error()


def test_relative_buckets():
    """Hand-worked: 8 buckets for both signs, reach 16: per sign 0, 1 exact and
    two logarithmic ranges split at 2 * sqrt(8) = 5.66."""
    m = api.relative_buckets(8, 16)
    at = lambda d: int(m[16 + d])  # noqa: E731
    assert [at(-d) for d in (0, 1, 2, 5, 6, 16)] == [0, 1, 2, 2, 3, 3]
    assert [at(d) for d in (1, 2, 5, 6, 16)] == [5, 6, 6, 7, 7]
    m = api.relative_buckets(8, 16, bidirectional=False)
    assert [int(m[16 - d]) for d in (0, 1, 2, 3, 4, 5, 6, 8, 11, 12, 16)] == [0, 1, 2, 3, 4, 4, 5, 6, 6, 7, 7]
    assert (m[17:] == 0).all()
    for bad in ((2, 16), (300, 400), (32, 8)):
        with pytest.raises(ValueError):
            api.relative_buckets(*bad)


def test_reference_generator_known_answers():
    """Known answers of Philox4x32-10 published with the generator."""
    from scored_reference import philox
    ones = np.uint64(0xFFFFFFFF)
    z = philox(np.zeros((1, 4), np.uint64), (0, 0))[0]
    assert [hex(int(v)) for v in z] == ["0x6627e8d5", "0xe169c58d", "0xbc57ac4c", "0x9b00dbd8"]
    f = philox(np.full((1, 4), ones), (0xFFFFFFFF, 0xFFFFFFFF))[0]
    assert [hex(int(v)) for v in f] == ["0x408f276d", "0x41c83b0e", "0xa20bc7c6", "0x6d5451fd"]


def test_dropout_refusals():
    L = api.lib()

    def call(x=4096, xs=8, r=None, rs=0, y=4096, ys=8, dtype=0, rows=2, cols=8, p=0.5):
        return L.fo_dropout_add(x, xs, r, rs, y, ys, dtype, rows, cols, p, 1, 1, None)

    for kw in ({"x": None}, {"y": None}, {"x": 4097}, {"r": 4098}, {"dtype": 7}, {"rows": -1}, {"cols": -1},
               {"rows": 1 << 40, "cols": 1 << 40}, {"p": -0.1}, {"p": 1.1}, {"p": float("nan")}, {"ys": 7}, {"xs": -8},
               {"r": 4096, "rs": -1}):
        assert call(**kw) == api.ERR_ARG and "dropout" in api.last_error(), kw
    assert call(rows=0) == api.OK and call(cols=0) == api.OK
