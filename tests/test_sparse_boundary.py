"""Argument checks of attention over selected key blocks (no GPU work), and pins of the 64-bit statement."""
import pytest
import torch

from tests import sparse_ref as R

A, STEP = 0x7F0000000000, 1 << 33        # fake, aligned, well separated addresses


@pytest.fixture(scope="module")
def aj():
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


BASE = dict(B=1, H=2, Lq=300, Lk=500, D=64)
SHAPES = [(dict(B=0), 2), (dict(H=0), 2), (dict(Lq=0), 2), (dict(Lk=-1), 2), (dict(D=96), 3), (dict(Lk=786433), 2),
          (dict(B=70000), 2), (dict(H=1 << 30), 2)]


def select(aj, topk=2, q=A, k=A + STEP, mask=A + 2 * STEP, index=A + 3 * STEP, tiles=A + 4 * STEP, ws=A + 5 * STEP, n=None, **kw):
    s = {**BASE, **kw}
    n = aj.attn_jvp_block_select_workspace_bytes(**s) if n is None else n
    return aj.attn_jvp_block_select(q, k, s["B"], s["H"], s["Lq"], s["Lk"], s["D"], topk, mask, index, tiles, ws, n, None)


def fwd(aj, flags=0, scale=0.1, **kw):
    p = dict(q=A, k=A + STEP, v=A + 2 * STEP, tq=A + 3 * STEP, tk=A + 4 * STEP, tv=A + 5 * STEP, index=A + 6 * STEP,
             tiles=A + 7 * STEP, order=None, o=A + 8 * STEP, to=A + 9 * STEP, lse=A + 10 * STEP, mu=None, **BASE)
    p.update(kw)
    return aj.attn_jvp_sparse_fwd(**p, scale=scale, flags=flags, cuda_stream=None)


def bwd(aj, n=None, scale=0.1, **kw):
    p = dict(d_o=A, q=A + STEP, k=A + 2 * STEP, v=A + 3 * STEP, o=A + 4 * STEP, lse=A + 5 * STEP, mask=A + 6 * STEP,
             index=A + 7 * STEP, tiles=A + 8 * STEP, order=None, dq=A + 9 * STEP, dk=A + 10 * STEP, dv=A + 11 * STEP, workspace=A + 12 * STEP,
             **BASE)
    p.update(kw)
    if n is None:
        n = aj.attn_jvp_sparse_bwd_workspace_bytes(*(p[m] for m in ("B", "H", "Lq", "Lk", "D")))
    return aj.attn_jvp_sparse_bwd(**p, scale=scale, workspace_bytes=n, cuda_stream=None)


@pytest.mark.parametrize("kw,code", SHAPES)
def test_shapes(aj, kw, code):
    assert select(aj, **kw) == code
    assert fwd(aj, **kw) == code
    assert bwd(aj, **kw) == code
    s = {**BASE, **kw}
    assert aj.attn_jvp_block_select_workspace_bytes(**s) == aj.attn_jvp_sparse_bwd_workspace_bytes(**s) == 0
    if code == 2:
        assert aj.attn_jvp_block_lists(A, s["B"], s["H"], s["Lq"], s["Lk"], A + STEP, A + 2 * STEP, None, None) == 2


def test_selection_refuses(aj):
    assert select(aj, topk=0) == 2
    for p in ("q", "k", "mask", "index", "tiles", "ws"):
        assert select(aj, **{p: None}) == 1
    assert select(aj, q=A + 2) == 4 and select(aj, index=A + 3 * STEP + 2) == 4 and select(aj, ws=A + 5 * STEP + 8) == 4
    assert select(aj, mask=A + 64) == 7 and select(aj, tiles=A + 3 * STEP) == 7
    assert select(aj, n=aj.attn_jvp_block_select_workspace_bytes(**BASE) - 1) == 12
    lists = aj.attn_jvp_block_lists
    assert lists(None, 1, 2, 300, 500, A, A + STEP, None, None) == 1
    assert lists(A, 1, 2, 300, 500, A + 1, A + STEP, None, None) == 4
    assert lists(A, 1, 2, 300, 500, A, A + STEP, None, None) == 7
    assert lists(A, 1, 2, 300, 500, A + STEP, A + 2 * STEP, A + 3 * STEP + 2, None) == 4
    assert lists(A, 1, 2, 300, 500, A + STEP, A + 2 * STEP, A + 2 * STEP, None) == 7


def test_forward_refuses(aj):
    for p in ("q", "k", "v", "tq", "tk", "tv", "index", "tiles", "o", "to", "lse"):
        assert fwd(aj, **{p: None}) == 1
    assert fwd(aj, flags=8) == 5
    assert fwd(aj, scale=float("nan")) == 6
    assert fwd(aj, k=A + STEP + 8) == 4 and fwd(aj, lse=A + 10 * STEP + 4) == 4
    assert fwd(aj, order=A + 6 * STEP + 2) == 4 and fwd(aj, order=A + 8 * STEP) == 7 and bwd(aj, order=A + 9 * STEP) == 7
    assert fwd(aj, o=A) == 7 and fwd(aj, to=A + 6 * STEP) == 7 and fwd(aj, mu=A + 8 * STEP) == 7


def test_backward_refuses(aj):
    for p in ("d_o", "q", "k", "v", "o", "lse", "mask", "index", "tiles", "dq", "dk", "dv", "workspace"):
        assert bwd(aj, **{p: None}) == 1
    assert bwd(aj, scale=float("inf")) == 6
    assert bwd(aj, dq=A + 9 * STEP + 8) == 4 and bwd(aj, workspace=A + 12 * STEP + 128) == 4
    assert bwd(aj, dq=A + STEP) == 7 and bwd(aj, dv=A + 10 * STEP) == 7 and bwd(aj, workspace=A + 6 * STEP) == 7
    assert bwd(aj, n=aj.attn_jvp_sparse_bwd_workspace_bytes(**BASE) - 1) == 12


def test_good_arguments_stop_at_the_device(aj):
    if torch.cuda.is_available():
        pytest.skip("would enqueue work on fake addresses")
    assert select(aj) in (8, 9) and fwd(aj) in (8, 9) and bwd(aj) in (8, 9)
    assert fwd(aj, flags=2, tq=None, tk=None, tv=None, to=None) in (8, 9)
    assert fwd(aj, flags=1, tk=None, tv=None, mu=A + 11 * STEP) in (8, 9)
    assert aj.attn_jvp_block_lists(A, 1, 2, 300, 500, A + STEP, A + 2 * STEP, None, None) in (8, 9)


def test_workspace_sizes(aj):
    # means of 3 query and 4 key blocks; lists of 4 key blocks over 3 query blocks, their lengths and order, counters, 384 padded
    # rows
    assert aj.attn_jvp_block_select_workspace_bytes(**BASE) == 2 * 64 * 8 * (3 + 4)
    assert aj.attn_jvp_sparse_bwd_workspace_bytes(**BASE) == 256 + 256 + 256 + 256 + 2 * 384 * 8


def test_python_layer_refuses_cpu_tensors(aj):
    q = torch.zeros(1, 200, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        aj.block_select(q, q, 1)
    with pytest.raises(ValueError):
        aj.block_selection(torch.ones(1, 2, 2, 2, dtype=torch.bool), 200, 200)


def test_layers_refuse_missing_tangents(aj):
    x = torch.zeros(1, 200, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="tangent"):
        aj.SparseAttentionCoreJVP(1)(x, x, x, withT=True)
    with pytest.raises(ValueError, match="tangent"):
        aj.SparseAttentionCoreJVP(1)((x, x), (x, x), x, withT=True)
    y = torch.zeros(1, 20, 64, dtype=torch.bfloat16)
    for a in ((y,), (y, (y, y)), ((y, y), y)):
        with pytest.raises(ValueError, match="tangent"):
            aj.AdaLNJVP(64)(*a, withT=True)


# ---- the 64-bit statement ----
def test_statement_with_every_block_is_attention(oracle):
    g = torch.Generator().manual_seed(0)
    q, k, v, tq, tk, tv, d_o = (torch.randn(1, L, 2, 64, generator=g).bfloat16() for L in (150, 200, 200, 150, 200, 200, 150))
    r = R.attention(q, k, v, torch.ones(1, 2, 2, 2, dtype=torch.bool), 0.125, tq, tk, tv, d_o)
    for h in range(2):
        args = [t[0, :, h].double().numpy() for t in (q, k, v, tq, tk, tv)]
        f = lambda a, b, c: torch.softmax(a @ b.T * 0.125, -1) @ c  # noqa: E731
        prim = tuple(torch.from_numpy(x) for x in args[:3])
        o, to = torch.func.jvp(f, prim, tuple(torch.from_numpy(x) for x in args[3:]))
        assert torch.allclose(r["o"][0][0, :, h], o, atol=1e-12) and torch.allclose(r["to"][0][0, :, h], to, atol=1e-12)
        grads = torch.func.vjp(f, *prim)[1](d_o[0, :, h].double())
        for n, w in zip(("dq", "dk", "dv"), grads):
            assert torch.allclose(r[n][0][0, :, h], w, atol=1e-12)


def test_statement_of_empty_rows_and_of_left_out_keys():
    g = torch.Generator().manual_seed(1)
    q, k, v, d_o = (torch.randn(1, L, 1, 64, generator=g).bfloat16() for L in (300, 260, 260, 300))
    mask = torch.tensor([[[[1, 0, 1], [0, 0, 0], [1, 0, 0]]]], dtype=torch.bool)
    r = R.attention(q, k, v, mask, 0.125, d_o=d_o)
    assert (r["o"][0][0, 128:256] == 0).all() and torch.isneginf(r["lse"][0][0, 0, 128:256]).all()
    assert (r["dk"][0][0, 128:256] == 0).all() and (r["dv"][0][0, 128:256] == 0).all() and (r["dq"][0][0, 128:256] == 0).all()
    kept = torch.cat([k[:, :128], k[:, 256:]], 1)
    want = torch.logsumexp(q[0, :128, 0].double() @ kept[0, :, 0].double().T * 0.125, -1)
    assert torch.allclose(r["lse"][0][0, 0, :128], want)


def test_statement_of_the_selection():
    """Two-token blocks would do; with whole blocks: constant blocks make the scores plain products."""
    q = torch.zeros(1, 256, 1, 64, dtype=torch.bfloat16)
    k = torch.zeros(1, 500, 1, 64, dtype=torch.bfloat16)
    q[0, :128, 0, 0], q[0, 128:, 0, 0] = 1.0, -1.0
    for j, c in enumerate((3.0, 5.0, 5.0, 1.0)):
        k[0, 128 * j:128 * (j + 1), 0, 0] = c
    m = R.top_mask(q, k, 2)[0, 0]
    assert m.tolist() == [[False, True, True, False], [True, False, False, True]]
    assert R.top_mask(q, k, 1)[0, 0].tolist() == [[False, True, False, False], [False, False, False, True]]
