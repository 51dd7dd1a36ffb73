"""Host side of the drafted-token and cache-page operators: no device needed."""
import ctypes
import math

import numpy as np
import pytest

from oracle import draft
from paper_2609_14237_b200 import binding as B


@pytest.fixture(scope="module", autouse=True)
def built():
    B.build()


SCALINGS = [("plain", {}), ("linear", dict(factor=4.0)), ("ntk", dict(factor=8.0)),
            ("bands", dict(factor=8.0, original_context=8192.0)),
            ("bands", dict(factor=32.0, original_context=2048.0, low=2.0, high=16.0)),
            ("yarn", dict(factor=16.0, original_context=4096.0)),
            ("yarn", dict(factor=4.0, original_context=100.0, low=0.5, high=8.0))]


@pytest.mark.parametrize("rot", [2, 18, 64, 128, 256])
@pytest.mark.parametrize("scaling,kw", SCALINGS)
def test_rope_table_is_the_formula(rot, scaling, kw):
    if scaling == "ntk" and rot == 2:
        with pytest.raises(B.OpwError):
            B.opw_rope_table(rot, scaling=scaling, **kw)
        return
    got = B.opw_rope_table(rot, theta=500000.0, scaling=scaling, **kw)
    names = {"original_context": "original"}
    want = draft.frequencies(rot, 500000.0, scaling, **{names.get(k, k): v for k, v in kw.items()})
    # a handful of 64-bit operations and one power on either side
    assert np.allclose(np.array(got[:-1]) * 2 * math.pi, want, rtol=1e-13, atol=0)
    amp = 1 + 0.1 * math.log(kw["factor"]) if scaling == "yarn" else 1.0
    assert math.isclose(got[-1], amp, rel_tol=1e-15)
    assert B.opw_rope_table(rot, scaling=scaling, amplitude=0.25, **kw)[-1] == 0.25


@pytest.mark.parametrize("kw", [dict(rotary_dim=0), dict(rotary_dim=7), dict(rotary_dim=258), dict(theta=1.0), dict(theta=math.inf),
                                dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=math.nan),
                                dict(scaling="bands", factor=2.0), dict(scaling="yarn", factor=2.0, original_context=-1.0),
                                dict(scaling="yarn", factor=2.0, original_context=100.0, low=4.0, high=2.0),
                                dict(amplitude=-1.0)])
def test_rope_table_refuses(kw):
    with pytest.raises(B.OpwError) as e:
        B.opw_rope_table(**{"rotary_dim": 64, **kw})
    assert e.value.status == B.OPW_ERR_INVALID_ARG


def test_rope_table_checks_its_struct():
    L, out = B.lib(), (ctypes.c_double * 33)()
    good = B.RopeConfig(ctypes.sizeof(B.RopeConfig), 64, 0, 0, 1e4, 1.0, 0.0, 0.0, 0.0, 0.0)
    assert L.opw_rope_table(ctypes.byref(good), out) == B.OPW_OK
    for field, value in (("struct_size", 8), ("scaling", 5), ("scaling", -1), ("reserved", 1)):
        bad = B.RopeConfig.from_buffer_copy(good)
        setattr(bad, field, value)
        assert L.opw_rope_table(ctypes.byref(bad), out) == B.OPW_ERR_INVALID_ARG
    assert L.opw_rope_table(None, out) == L.opw_rope_table(ctypes.byref(good), None) == B.OPW_ERR_INVALID_ARG


def test_tree_mask_and_depth():
    mask, depth = B.opw_tree_mask([-1, 0, 0, 1, -1, 4, 3])
    assert mask == [0b1, 0b11, 0b101, 0b1011, 0b10000, 0b110000, 0b1001011] and depth == [0, 1, 1, 2, 0, 1, 3]
    mask, depth = B.opw_tree_mask([i - 1 for i in range(64)])
    assert mask == [(2 << i) - 1 for i in range(64)] and depth == list(range(64))
    for bad in ([0], [-2], [-1, 1], [-1, 0, 5], [], [i - 1 for i in range(65)]):
        with pytest.raises(B.OpwError):
            B.opw_tree_mask(bad)


def test_null_handles_are_refused():
    L, h = B.lib(), ctypes.c_void_p()
    one = (ctypes.c_int32 * 1)(0)
    assert L.opw_tree_attn_workspace_bytes(None, 8) == 0
    assert L.opw_tree_attn_create(None, 8, 0, 256, 1 << 30, ctypes.byref(h)) == B.OPW_ERR_INVALID_ARG and h.value is None
    assert L.opw_tree_attention(None, 0, 1, 4, *[16] * 7, None, None) == B.OPW_ERR_INVALID_ARG
    assert L.opw_tree_attn_destroy(None) == B.OPW_OK
    assert L.opw_rope_append(None, 0, 1, 64, 0, 16, 16, 64, 16, 64, 16, 64, 16, 16, 16, 1, 16, 16, None) == B.OPW_ERR_INVALID_ARG
    assert L.opw_kv_commit(None, one, 1, 1, 4, 16, 16, 16, 16, None, None) == B.OPW_ERR_INVALID_ARG
    assert L.opw_kv_fork(None, one, 1, 1, 16, 16, 16, 16, 1, 16, 16, None) == B.OPW_ERR_INVALID_ARG
    assert L.opw_kv_release(None, 1, 16, None, 1, 16, 16, 1, None) == B.OPW_ERR_INVALID_ARG
    assert L.opw_kv_free_pages(None, 16, 1, 16, 1, 16, None) == B.OPW_ERR_INVALID_ARG


def test_the_oracle_of_tree_attention_is_softmax_over_what_a_node_sees():
    """A chain over an empty context is causal attention; a node that sees itself only returns its own value."""
    import oracle

    rng = np.random.default_rng(5)
    T, D = 5, 64
    x = lambda *s: oracle.f32_to_bf16_bits(rng.standard_normal(s).astype(np.float32))  # noqa: E731
    pool, table = np.zeros(oracle.pool_elems(2, 1, 16, D), np.uint16), np.array([[1, -1]], np.int32)
    k, v, q = x(T, 1, D), x(T, 1, D), x(1, T, 2, D)
    draft.append_rows(pool, 1, D, [0] * T, list(range(T)), table, k, v)
    f = oracle.bf16_bits_to_f64
    chain = np.array([[(2 << i) - 1 for i in range(T)]], np.uint64)
    out, lse, _, _ = draft.tree_attention(pool, 2, 1, D, q, chain, np.arange(T)[None], [0], [T], table)
    for i in range(T):
        p = np.exp(f(k)[:i + 1, 0] @ f(q)[0, i, 1] / 8.0)
        assert np.allclose(out[0, i, 1], p @ f(v)[:i + 1, 0] / p.sum(), rtol=1e-12, atol=1e-12)
        assert math.isclose(lse[0, i, 1], math.log(p.sum()), rel_tol=1e-12, abs_tol=1e-12)
    own = np.array([[1 << i for i in range(T)]], np.uint64)
    out, _, _, _ = draft.tree_attention(pool, 2, 1, D, q, own, np.arange(T)[None], [0], [T], table)
    assert (out[0, :, 0] == f(v)[:, 0]).all()
    # a window of one position leaves the node itself, however deep it stands
    out, _, _, _ = draft.tree_attention(pool, 2, 1, D, q, chain, np.arange(T)[None], [0], [T], table, window=1)
    assert (out[0, :, 0] == f(v)[:, 0]).all()


def test_the_oracle_of_rotation_keeps_norms_and_position_differences():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((3, 2, 64))
    for layout in ("half", "interleaved"):
        f = draft.frequencies(32)
        assert (draft.rotate(x, np.zeros(3), f, layout) == x).all()
        y = draft.rotate(x, np.array([5, 77, 123456]), f, layout)
        assert np.allclose((y ** 2).sum(-1), (x ** 2).sum(-1)) and (y[:, :, 32:] == x[:, :, 32:]).all()
        dots = [(draft.rotate(x[:1], np.array([m]), f, layout) * draft.rotate(x[1:2], np.array([n]), f, layout)).sum()
                for m, n in ((3, 10), (1003, 1010))]
        assert math.isclose(dots[0], dots[1], rel_tol=1e-9)
