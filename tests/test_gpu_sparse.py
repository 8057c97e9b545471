"""Attention over selected key blocks on the GPU: selection, forward, tangents, gradients, against the 64-bit statement in
tests/sparse_ref.py (which also derives the tolerances)."""
import pytest
import torch

from paper_2510_08431_b200 import synth
from tests import sparse_differences as F
from tests import sparse_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def aj():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2510_08431_b200 import build
    build.build_library()
    import paper_2510_08431_b200 as aj
    aj.load()
    return aj


def inputs(B, H, Lq, Lk, D, seed=0):
    x = {n: t.cuda() for n, t in synth.make_inputs(B, H, Lq, Lk, D, 1.0, 0.7, seed=seed + Lq + 3 * Lk).items()}
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    x["d_o"] = torch.randn(B, Lq, H, D, generator=g, device="cuda").bfloat16()
    return x


def make_mask(kind, B, H, n_q, n_k, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed + 17 * n_q + n_k)
    r = torch.rand(B, H, n_q, n_k, generator=g, device="cuda")
    if kind == "all":
        return torch.ones_like(r, dtype=torch.bool)
    if kind == "none":
        return torch.zeros_like(r, dtype=torch.bool)
    if kind == "last":                       # only the ragged last key block
        m = torch.zeros_like(r, dtype=torch.bool)
        m[..., -1] = True
        return m
    if kind == "one":                        # one key block per row, and some rows none
        return (torch.nn.functional.one_hot(r.argmax(-1), n_k).bool()) & (r[..., :1] > 0.2)
    m = r < 0.4                              # "mixed": lengths from none to all, whole rows and columns empty
    m[:, :, ::3] &= r[:, :, ::3, :1] < 0.5
    m[:, :, :, 0] = False
    m[:, 0, n_q // 2] = False
    m[:, -1, n_q - 1] = True
    return m


def no_timeout(aj):
    torch.cuda.synchronize()
    st = aj.attn_jvp_device_status()
    assert st == 0, (aj.attn_jvp_strerror(st), aj.attn_jvp.attn_jvp_debug_timeout_info())


def run_all(aj, x, sel, D, scale=None):
    s = D ** -0.5 if scale is None else scale
    got = {}
    got["o"], none, got["lse"] = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, fwd_only=True, scale=scale)
    no_timeout(aj)
    assert none is None
    ref = R.attention(x["q"], x["k"], x["v"], sel.mask, s, x["tq"], x["tk"], x["tv"], x["d_o"])
    for n in got:
        R.check(n, got[n], ref[n])
    o, to, lse, mu = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, x["tq"], x["tk"], x["tv"], scale=scale, return_mu=True)
    no_timeout(aj)
    for n, g in dict(o=o, to=to, lse=lse, mu=mu).items():
        R.check(n, g, ref[n])
    free = R.attention(x["q"], x["k"], x["v"], sel.mask, s, x["tq"])
    o, to, lse, mu = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, x["tq"], scale=scale, return_mu=True)
    no_timeout(aj)
    for n, g in dict(o=o, to=to, lse=lse, mu=mu).items():
        R.check(n + " (constant context)", g, free[n])
    dq, dk, dv = aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], got["o"], got["lse"], sel, scale=scale)
    no_timeout(aj)
    for n, g in dict(dq=dq, dk=dk, dv=dv).items():
        R.check(n, g, ref[n])


SIZES = [(1, 1), (1, 333), (64, 65), (128, 128), (129, 64), (200, 333), (333, 192), (517, 1000), (1000, 257)]


@pytest.mark.parametrize("Lq,Lk", SIZES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("kind", ["mixed", "all", "one", "last", "none"])
def test_given_masks(aj, Lq, Lk, D, kind):
    B, H = 2, 3
    sel = aj.block_selection(make_mask(kind, B, H, R.blocks(Lq), R.blocks(Lk)), Lq, Lk)
    run_all(aj, inputs(B, H, Lq, Lk, D), sel, D)


@pytest.mark.parametrize("D", [64, 128])
def test_more_items_than_multiprocessors(aj, D):
    """Persistent CTAs walk several items of different lengths, empty ones among them."""
    B, H, Lq, Lk = 2, 13, 1100, 1500
    sel = aj.block_selection(make_mask("mixed", B, H, R.blocks(Lq), R.blocks(Lk)), Lq, Lk)
    run_all(aj, inputs(B, H, Lq, Lk, D), sel, D)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("scale", [0.0, -0.11, 0.3])
def test_scales(aj, D, scale):
    sel = aj.block_selection(make_mask("mixed", 1, 2, 3, 4), 300, 450)
    run_all(aj, inputs(1, 2, 300, 450, D), sel, D, scale=scale)


@pytest.mark.parametrize("D", [64, 128])
def test_long_rows(aj, D):
    """Many key blocks per row: every ring and barrier goes round many times."""
    sel = aj.block_selection(make_mask("all", 1, 2, 3, 40), 300, 5000)
    run_all(aj, inputs(1, 2, 300, 5000, D), sel, D)
    sel = aj.block_selection(make_mask("mixed", 1, 2, 40, 3), 5000, 300)
    run_all(aj, inputs(1, 2, 5000, 300, D), sel, D)


def test_all_blocks_is_the_dense_kernel(aj):
    """With every block kept the JVP takes the tiles of attention_jvp in its order, and the same arithmetic."""
    for D in (64, 128):
        x = inputs(1, 2, 640, 1100, D)
        sel = aj.block_selection(make_mask("all", 1, 2, 5, 9), 640, 1100)
        a = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, x["tq"], x["tk"], x["tv"])
        b = aj.attention_jvp(x["q"], x["k"], x["v"], x["tq"], x["tk"], x["tv"])
        no_timeout(aj)
        for u, v in zip(a, b):
            assert torch.equal(u, v)


@pytest.mark.parametrize("B,H,Lq,Lk,D,topk", [(1, 2, 200, 333, 64, 2), (2, 3, 1000, 1300, 128, 4), (1, 1, 1, 1, 64, 1),
                                              (1, 2, 130, 70, 128, 5), (1, 5, 4100, 8000, 64, 17), (2, 1, 65, 129, 128, 1)])
def test_selection_by_block_means(aj, B, H, Lq, Lk, D, topk):
    x = inputs(B, H, Lq, Lk, D)
    sel = aj.block_select(x["q"], x["k"], topk)
    want = R.top_mask(x["q"], x["k"], topk)
    assert torch.equal(sel.mask, want)
    lists(sel)


def lists(sel):
    """index and tiles say what the mask says."""
    n = sel.mask.shape[-1]
    tail = sel.Lk - (n - 1) * 128
    count = sel.mask.sum(-1)
    short = sel.mask[..., -1] if tail <= 64 else torch.zeros_like(sel.mask[..., -1])
    assert torch.equal(sel.tiles.long(), 2 * count - short.long())
    want = torch.sort(sel.mask.to(torch.uint8), dim=-1, descending=True, stable=True).indices
    live = torch.arange(n, device="cuda") < count[..., None]
    assert torch.equal(sel.index[live].long(), want[live])
    if sel.order is not None:
        # windows of 888 consecutive rows, the longest lists first, equal ones as they lie
        tiles = sel.tiles.flatten().long()
        expected = [w + torch.sort(tiles[w:w + 888], descending=True, stable=True).indices for w in range(0, tiles.numel(), 888)]
        assert torch.equal(sel.order.flatten().long(), torch.cat(expected))


@pytest.mark.parametrize("n_k", [1, 31, 32, 33, 100])
@pytest.mark.parametrize("tail", [1, 64, 65, 128])
def test_lists_of_a_mask(aj, n_k, tail):
    Lk = (n_k - 1) * 128 + tail
    for kind in ("mixed", "none", "all", "last"):
        lists(aj.block_selection(make_mask(kind, 2, 3, 5, n_k), 600, Lk))


@pytest.mark.parametrize("B,H,Lq,Lk,D", [(1, 3, 12700, 900, 64), (2, 10, 6000, 700, 128), (3, 7, 5700, 5700, 64)])
def test_order_of_work(aj, B, H, Lq, Lk, D):
    """More rows than a window, and partial last rounds of either direction: the same bits in either order of work."""
    x = inputs(B, H, Lq, Lk, D)
    sel = aj.block_selection(make_mask("mixed", B, H, R.blocks(Lq), R.blocks(Lk)), Lq, Lk)
    lists(sel)

    def path(s):
        o, to, lse, mu = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], s, x["tq"], x["tk"], x["tv"], return_mu=True)
        f, _, fl = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], s, fwd_only=True)
        res = (o, to, lse, mu, f, fl) + aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], f, fl, s)
        no_timeout(aj)
        return res

    for u, v in zip(path(sel), path(sel._replace(order=None))):
        assert torch.equal(u, v)


def test_ties_go_to_the_lower_block(aj):
    """Equal key blocks have equal scores whatever the order of the sums; of them the first ones are kept."""
    x = inputs(1, 2, 256, 128 * 70, 64)
    k = x["k"].view(1, 70, 128, 2, 64)
    k[:, 5:60] = k[:, 5:6]
    for topk in (1, 7, 33, 69):
        sel = aj.block_select(x["q"], x["k"], topk)
        assert torch.equal(sel.mask, R.top_mask(x["q"], x["k"], topk)), topk
        assert (sel.mask.sum(-1) == topk).all()
        lists(sel)
    zero = torch.zeros_like(x["k"])
    sel = aj.block_select(x["q"], zero, 3)
    assert (sel.mask[..., :3]).all() and not sel.mask[..., 3:].any()


def test_ties_of_many_key_blocks(aj):
    """A row of equal scores (padding) longer than a lane holds in registers: the first ones, in one pass over the row."""
    q = torch.randn(1, 128 * 20, 1, 64, device="cuda").bfloat16()
    k = torch.zeros(1, 128 * 6144, 1, 64, device="cuda", dtype=torch.bfloat16)
    k[:, 128 * 6000 : 128 * 6002] = 1.0                                   # above zero or below it, by the sign of the query's sum
    sel = aj.block_select(q, k, 700)
    high = q.view(20, 128 * 64).double().sum(1) > 0
    for i in range(20):
        want = torch.cat([torch.arange(698), torch.tensor([6000, 6001])]) if high[i] else torch.arange(700)
        assert torch.equal(sel.mask[0, 0, i].nonzero()[:, 0].cpu(), want)
    lists(sel)


@pytest.mark.parametrize("n_k", [300, 3300])
def test_selection_of_many_key_blocks(aj, n_k):
    """More key blocks than a lane holds in registers, and more than eight rows have room for."""
    q = torch.randn(1, 300, 1, 64, device="cuda").bfloat16()
    k = torch.randn(1, n_k * 128 - 37, 1, 64, device="cuda").bfloat16()
    sel = aj.block_select(q, k, 100)
    assert torch.equal(sel.mask, R.top_mask(q, k, 100))
    lists(sel)


def test_selection_of_tiny_and_huge_values(aj):
    """bf16 subnormals and the largest values go through the means exactly."""
    q = torch.randn(1, 256, 1, 64, device="cuda")
    k = torch.randn(1, 1280, 1, 64, device="cuda")
    for f in (1e-39, 1e37):
        qq, kk = (q * f).bfloat16(), k.bfloat16()
        assert torch.equal(aj.block_select(qq, kk, 4).mask, R.top_mask(qq, kk, 4))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n_k", [6, 300])
@pytest.mark.parametrize("bad", ["nan", "inf", "-inf", "both", "nan_and_inf", "query", "all_queries"])
def test_selection_with_infinities_and_nan(aj, D, n_k, bad):
    """They follow IEEE arithmetic through means and scores, and NaN scores come first, ties to the lower block, as a stable
    descending sort has them (the reference sorts on the CPU, which orders NaN by value and not by sign)."""
    B, H, Lq, Lk = 2, 2, 400, n_k * 128 - 50
    x = inputs(B, H, Lq, Lk, D)
    q, k = x["q"], x["k"]
    inf, nan = float("inf"), float("nan")
    if bad == "nan":
        k[0, 128 * 4 + 77, 1, 5] = nan
        k[1, 128 * 2, 0, D - 1] = -nan
    elif bad == "inf":
        k[0, 130, 0, 9] = inf
        k[1, Lk - 1, 1, 0] = inf
    elif bad == "-inf":
        k[:, 128 * 3 + 127, :, D // 2] = -inf
    elif bad == "both":
        k[0, 128, 1, 1], k[0, 255, 1, 1] = inf, -inf          # one channel's mean is NaN
        k[1, 128, 1, 1], k[1, 300, 1, 2] = inf, -inf          # two blocks, each infinite
    elif bad == "nan_and_inf":
        k[:, 10, :, 3], k[:, 140, :, 3], k[:, 500, :, 7] = nan, inf, nan
    elif bad == "query":
        q[0, 129, 0, 2], q[1, 399, 1, 8] = nan, inf
    else:
        q[:, :, :, 4] = inf
        k[:, 128:256, :, 4] = 0.0                             # 0 times infinity
    for topk in (1, 2, 5):
        sel = aj.block_select(q, k, topk)
        assert torch.equal(sel.mask.cpu(), R.top_mask(q.cpu(), k.cpu(), topk)), topk
        assert (sel.mask.sum(-1) == topk).all()
        lists(sel)


def test_select_attend_and_train_together(aj):
    """The path as it is used: selection, forward, gradients; two passes give the same bits."""
    B, H, Lq, Lk, D = 1, 4, 2100, 2500, 128
    x = inputs(B, H, Lq, Lk, D)
    sel = aj.block_select(x["q"], x["k"], 5)
    run_all(aj, x, sel, D)

    def once():
        s = aj.block_select(x["q"], x["k"], 5)
        o, _, lse = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], s, fwd_only=True)
        return (o, lse) + aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, s)

    for u, v in zip(once(), once()):
        assert torch.equal(u, v)


def test_gradients_against_differences(aj):
    """<gradient, direction> = central difference of the 64-bit loss; the gradients' own tolerances, summed, bound the rest."""
    B, H, Lq, Lk, D = 1, 1, 150, 300, 64
    x = inputs(B, H, Lq, Lk, D)
    mask = make_mask("all", B, H, 2, 3)
    mask[0, 0, 0, 1] = False
    sel = aj.block_selection(mask, Lq, Lk)
    o, _, lse = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, fwd_only=True)
    grads = aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, sel)
    ref = R.attention(x["q"], x["k"], x["v"], mask, D ** -0.5, d_o=x["d_o"])
    keep = mask.repeat_interleave(128, 2)[0, 0, :Lq].repeat_interleave(128, 1)[:, :Lk]

    def loss(e, n, direction):
        a = {m: x[m].double()[0, :, 0] for m in "qkv"}
        a[n] = a[n] + e * direction
        S = torch.where(keep, a["q"] @ a["k"].T * D ** -0.5, -float("inf"))
        return ((torch.softmax(S, -1) @ a["v"]) * x["d_o"].double()[0, :, 0]).sum()

    g = torch.Generator(device="cuda").manual_seed(5)
    for n, grad in zip("qkv", grads):
        d = torch.randn(x[n].shape[1], D, generator=g, device="cuda", dtype=torch.float64)
        e = 1e-4
        want = (loss(e, n, d) - loss(-e, n, d)) / (2 * e)
        got = (grad.double()[0, :, 0] * d).sum()
        assert abs(got - want) <= (ref["d" + n][1][0, :, 0] * d.abs()).sum() + 1e-6 * abs(want)


@pytest.mark.parametrize("D,scale", [(64, None), (128, None), (64, -0.2)])
def test_gradients_along_their_own_directions(aj, D, scale):
    """<gradient, direction> = central difference of the 64-bit loss, with a tolerance that a wrong gradient exceeds
    (tests/sparse_differences.py; tests/test_sparse_differences.py shows which mistakes it finds)."""
    B, H, Lq, Lk = 2, 2, 150, 300
    x = inputs(B, H, Lq, Lk, D)
    mask = make_mask("all", B, H, 2, 3)
    mask[:, :, 0, 1] = False
    mask[0, 1, 1, 2] = False
    sel = aj.block_selection(mask, Lq, Lk)
    o, _, lse = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, fwd_only=True, scale=scale)
    grads = aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, sel, scale=scale)
    no_timeout(aj)
    rows = F.compare(dict(zip("qkv", grads)), x, mask, D ** -0.5 if scale is None else scale)
    assert F.passes(rows) == {"q", "k", "v"}, rows


def test_rows_behind_the_last_are_left_alone(aj):
    """Outputs end where the tensors end, whatever the last block's rows hold."""
    B, H, Lq, Lk, D = 1, 2, 130, 200, 128
    x = inputs(B, H, Lq, Lk, D)
    sel = aj.block_selection(make_mask("all", B, H, 2, 2), Lq, Lk)
    nq, nk, pad = B * Lq * H * D, B * Lk * H * D, 128 * H * D
    o, to, dq = (torch.full((nq + pad,), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(3))
    dk, dv = (torch.full((nk + pad,), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    lse = torch.full((B * H * Lq + 256,), 3.0, device="cuda")
    st = torch.cuda.current_stream().cuda_stream
    assert aj.attn_jvp_sparse_fwd(x["q"], x["k"], x["v"], x["tq"], x["tk"], x["tv"], sel.index, sel.tiles, sel.order, o, to, lse, None, B, H,
                                  Lq, Lk, D, 0.1, 0, st) == 0
    ws = torch.empty(aj.attn_jvp_sparse_bwd_workspace_bytes(B, H, Lq, Lk, D), dtype=torch.uint8, device="cuda")
    assert aj.attn_jvp_sparse_bwd(x["d_o"], x["q"], x["k"], x["v"], o, lse, sel.mask, sel.index, sel.tiles, sel.order, dq, dk, dv, B, H, Lq,
                                  Lk, D, 0.1, ws, ws.numel(), st) == 0
    no_timeout(aj)
    for t, n in ((o, nq), (to, nq), (dq, nq), (dk, nk), (dv, nk), (lse, B * H * Lq)):
        assert (t[n:] == 3.0).all() and not (t[:n] == 3.0).all()


@pytest.mark.parametrize("D", [64, 128])
def test_nothing_is_read_where_nothing_is_kept(aj, D):
    """NaN and infinities in a query block without keys and in a key block that nobody kept reach no result."""
    B, H, Lq, Lk = 1, 2, 400, 500
    mask = make_mask("all", B, H, 4, 4)
    mask[:, :, 1] = False
    mask[..., 2] = False
    sel = aj.block_selection(mask, Lq, Lk)

    def path(x):
        o, to, lse, mu = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, x["tq"], x["tk"], x["tv"], return_mu=True)
        free = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, x["tq"], return_mu=True)
        f, _, fl = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, fwd_only=True)
        res = dict(o=o, to=to, lse=lse, mu=mu, free_to=free[1], free_mu=free[3], f=f, fl=fl)
        res.update(zip(("dq", "dk", "dv"), aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], f, fl, sel)))
        no_timeout(aj)
        return res

    x = inputs(B, H, Lq, Lk, D)
    want = path(x)
    for n, bad in (("q", float("nan")), ("tq", float("inf")), ("d_o", float("nan"))):
        x[n][:, 128:256] = bad
    for n, bad in (("k", float("nan")), ("v", float("inf")), ("tk", float("-inf")), ("tv", float("nan"))):
        x[n][:, 256:384] = bad
    got = path(x)
    for n in want:
        assert torch.equal(got[n], want[n]), n
    for n in ("o", "to", "free_to", "f", "dq"):
        assert not got[n][:, 128:256].any(), n
    assert not got["mu"][:, :, 128:256].any() and (got["lse"][:, :, 128:256] == -float("inf")).all()
    assert not got["dk"][:, 256:384].any() and not got["dv"][:, 256:384].any()


@pytest.mark.parametrize("D", [64, 128])
def test_a_nan_in_one_query_reaches_its_gradients(aj, D):
    """P of a query with a NaN is NaN for every key it keeps, whichever row of its block it is: dQ of the row, dK and dV of its
    key blocks show it, and nothing else does."""
    B, H, Lq, Lk = 1, 1, 300, 400
    mask = torch.tensor([[[[1, 0, 1, 1], [0, 1, 0, 1], [1, 1, 1, 1]]]], dtype=torch.bool, device="cuda")
    sel = aj.block_selection(mask, Lq, Lk)
    for row in [128 + r for r in range(20)] + [128 + 126, 128 + 127]:
        x = inputs(B, H, Lq, Lk, D)
        x["q"][0, row, 0, 3] = float("nan")
        o, _, lse = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, fwd_only=True)
        dq, dk, dv = aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, sel)
        no_timeout(aj)
        kept = mask[0, 0, 1].repeat_interleave(128)[:Lk]
        assert dq[0, row].isnan().all() and dq.isnan().sum() == D, row
        for n, g in (("dk", dk), ("dv", dv)):
            assert g[0, kept].isnan().all() and g[0, ~kept].isfinite().all(), (n, row)


def test_outputs_between_sectors_and_given_buffers(aj):
    """Gradients 16 bytes off a 32-byte boundary, outputs and workspaces of the caller: the same bits."""
    B, H, Lq, Lk, D = 1, 3, 300, 450, 64
    x = inputs(B, H, Lq, Lk, D)
    sel = aj.block_select(x["q"], x["k"], 2)
    ws = torch.empty(aj.attn_jvp_block_select_workspace_bytes(B, H, Lq, Lk, D), dtype=torch.uint8, device="cuda")
    for u, v in zip(aj.block_select(x["q"], x["k"], 2, workspace=ws)[:1], sel[:1]):
        assert torch.equal(u, v)
    o, _, lse = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, fwd_only=True)
    mine = (torch.empty_like(o), None, torch.empty_like(lse))
    res = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, fwd_only=True, out=mine)
    assert res[0].data_ptr() == mine[0].data_ptr() and torch.equal(res[0], o) and torch.equal(res[2], lse)
    need = aj.attn_jvp_sparse_bwd_workspace_bytes(B, H, Lq, Lk, D)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    want = aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, sel)
    for u, v in zip(aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, sel, workspace=ws), want):
        assert torch.equal(u, v)
    outs = [torch.full((w.numel() + 16,), 5.0, dtype=torch.bfloat16, device="cuda") for w in want]
    assert all(t.data_ptr() % 32 == 0 for t in outs)
    assert aj.attn_jvp_sparse_bwd(x["d_o"], x["q"], x["k"], x["v"], o, lse, sel.mask, sel.index, sel.tiles, sel.order, *(t[8:] for t in outs),
                                  B, H, Lq, Lk, D, D ** -0.5, ws, need, torch.cuda.current_stream().cuda_stream) == 0
    no_timeout(aj)
    for t, w in zip(outs, want):
        assert torch.equal(t[8:w.numel() + 8], w.reshape(-1)) and (t[:8] == 5.0).all() and (t[w.numel() + 8:] == 5.0).all()


def test_many_heads_and_batches_of_one_block(aj):
    """More work items than an SM draws in a lap, all short, across batches."""
    B, H, L, D = 40, 9, 70, 64
    x = inputs(B, H, L, L, D)
    sel = aj.block_select(x["q"], x["k"], 1)
    run_all(aj, x, sel, D)


def test_captured_and_replayed_on_a_side_stream(aj):
    """The whole path in a CUDA graph: selection, forward and gradients follow the inputs of the replay."""
    B, H, Lq, Lk, D = 1, 2, 700, 900, 64
    x, y = inputs(B, H, Lq, Lk, D), inputs(B, H, Lq, Lk, D, seed=9)

    def path(z):
        s = aj.block_select(z["q"], z["k"], 3)
        o, to, lse = aj.sparse_attention_jvp(z["q"], z["k"], z["v"], s, z["tq"], z["tk"], z["tv"])
        f, _, fl = aj.sparse_attention_jvp(z["q"], z["k"], z["v"], s, fwd_only=True)
        return (s.mask, o, to, lse) + aj.sparse_attention_backward(z["d_o"], z["q"], z["k"], z["v"], f, fl, s)

    want = path(y)
    path(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = path(x)
    for n in x:
        x[n].copy_(y[n])
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        graph.replay()
    no_timeout(aj)
    for u, v in zip(got, want):
        assert torch.equal(u, v)


def test_two_streams_at_once(aj):
    """Independent calls on two streams (each with its own selection and workspace) do not meet."""
    xs = [inputs(1, 3, 900, 1100, 128, seed=s) for s in (0, 4)]

    def path(z):
        s = aj.block_select(z["q"], z["k"], 4)
        o, _, lse = aj.sparse_attention_jvp(z["q"], z["k"], z["v"], s, fwd_only=True)
        return (o, lse) + aj.sparse_attention_backward(z["d_o"], z["q"], z["k"], z["v"], o, lse, s)

    want = [path(z) for z in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for z, st in zip(xs, streams):
        with torch.cuda.stream(st):
            got.append([path(z) for _ in range(3)])
    no_timeout(aj)
    for w, runs in zip(want, got):
        for r in runs:
            for u, v in zip(r, w):
                assert torch.equal(u, v)


def test_python_layer_refuses(aj):
    x = inputs(1, 2, 200, 300, 64)
    sel = aj.block_selection(make_mask("all", 1, 2, 2, 3), 200, 300)
    with pytest.raises(ValueError):
        aj.block_selection(sel.mask, 300, 300)                          # blocks and lengths do not agree
    with pytest.raises(ValueError):
        aj.block_selection(sel.mask.int(), 200, 300)
    with pytest.raises(ValueError):
        aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel.mask, fwd_only=True)
    with pytest.raises(ValueError):
        aj.sparse_attention_jvp(x["q"][:, :100].contiguous(), x["k"], x["v"], sel, fwd_only=True)
    with pytest.raises(ValueError):
        aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, x["tq"], x["tk"])
    with pytest.raises(ValueError):
        aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel)
    with pytest.raises(aj.AttnJvpError) as e:
        aj.block_select(x["q"], x["k"], 0)
    assert e.value.code == 2
    o, _, lse = aj.sparse_attention_jvp(x["q"], x["k"], x["v"], sel, fwd_only=True)
    need = aj.attn_jvp_sparse_bwd_workspace_bytes(1, 2, 200, 300, 64)
    with pytest.raises(aj.AttnJvpError) as e:
        aj.sparse_attention_backward(x["d_o"], x["q"], x["k"], x["v"], o, lse, sel,
                                     workspace=torch.empty(need - 1, dtype=torch.uint8, device="cuda"))
    assert e.value.code == 12
