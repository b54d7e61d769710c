"""Verification of drafted tokens on the GPU against the walk written out in float64
(drafts_ref): paths, counts and tokens have to be equal."""
import random

import pytest
import torch

import drafts_ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def drafts(gpu_lib):
    from paper_2509_25689_amd import drafts
    return drafts


def _tree(rng, n, shape, wide=4):
    if shape == "chain":
        return list(range(-1, n - 1))
    if shape == "star":
        return [-1] + [0] * (n - 1)
    return [-1] + [rng.randint(max(0, i - wide), i - 1) for i in range(1, n)]


def _world(seed, sizes, V, shape, sampled, keep=0.6, sharp=2.0):
    rng, g = random.Random(seed), torch.Generator().manual_seed(seed)
    trees = [_tree(rng, n, shape) if n else [] for n in sizes]
    T = sum(sizes)
    logits = sharp * torch.randn((T, V), generator=g)
    target, draft = torch.softmax(logits, -1), torch.softmax(logits + torch.randn((T, V), generator=g), -1)
    cu = torch.tensor([0] + sizes).cumsum(0).int()
    tokens, at = [], 0
    for t in trees:
        for i, p in enumerate(t):
            row = draft[at + max(p, 0)]
            tokens.append(int(row.topk(min(3, V)).indices[rng.randrange(min(3, V))]) if rng.random() < 0.8 else rng.randrange(V))
        at += len(t)
    return dict(trees=trees, tokens=torch.tensor(tokens, dtype=torch.int32), parents=torch.tensor([p for t in trees for p in t], dtype=torch.int32),
                cu=cu, target=target, draft=draft if sampled else None, uniform=torch.rand(T, generator=g) * keep, last=torch.rand(len(sizes), generator=g))


def _cuda(w):
    return {k: v.cuda() if isinstance(v, torch.Tensor) else v for k, v in w.items()}


def _run(drafts, w, max_new, **kw):
    return drafts.verify(w["tokens"], w["parents"], w["cu"], w["target"], w["draft"], w["uniform"], w["last"], max_new=max_new, **kw)


def _expect(w, max_new):
    out = []
    cu = w["cu"].tolist()
    target = w["target"].double().numpy()
    draft = None if w["draft"] is None else w["draft"].double().numpy()
    for r in range(len(cu) - 1):
        a, b = cu[r], cu[r + 1]
        if a == b:
            out.append(([], []))
            continue
        out.append(drafts_ref.verify_one(w["tokens"][a:b].tolist(), w["parents"][a:b].tolist(), target[a:b], None if draft is None else draft[a:b],
                                         w["uniform"][a:b].double().tolist(), float(w["last"][r].double())))
    pad = lambda v: v + [-1] * (max_new - len(v))  # noqa: E731
    return [pad(p) for p, _ in out], [len(p) for p, _ in out], [pad(t) for _, t in out]


def _check(drafts, w, max_new=None, **kw):
    max_new = max_new or int((w["cu"][1:] - w["cu"][:-1]).max())
    path, counts, tokens = _run(drafts, _cuda(w), max_new, **kw)
    torch.cuda.synchronize()
    p, c, t = _expect(w, max_new)
    assert counts.tolist() == c and path.tolist() == p and tokens.tolist() == t
    return counts.tolist()


@pytest.mark.parametrize("sampled", [False, True])
@pytest.mark.parametrize("shape", ["chain", "tree", "star"])
@pytest.mark.parametrize("sizes,V", [([1], 1), ([2], 3), ([5, 1, 8, 3], 17), ([8] * 6, 1000), ([24, 9], 4097), ([6, 6], 12288), ([64], 300), ([7], 65537)])
def test_verify(drafts, sampled, shape, sizes, V):
    kept = [_check(drafts, _world(seed, sizes, V, shape, sampled, keep=(0.3, 1.0, 0.02)[seed])) for seed in range(3)]
    assert all(c >= 1 for k in kept for c in k)


@pytest.mark.parametrize("sampled", [False, True])
def test_verify_sizes(drafts, sampled):
    """Requests without tokens, trees of 256 (the most), and a table wider than any."""
    sizes = [0, 256, 3, 0, 65, 128, 0]
    _check(drafts, _world(11, sizes, 50, "tree", sampled, keep=0.1))
    _check(drafts, _world(12, [0, 5, 0], 50, "tree", sampled), max_new=77)


@pytest.mark.parametrize("sampled", [False, True])
def test_verify_twins(drafts, sampled):
    """Siblings of the same token, more than one rejected: what the first takes the second does not get."""
    w = _world(13, [6, 6], 9, "star", sampled)
    w["tokens"][:] = torch.tensor([0, 4, 4, 4, 2, 4, 0, 1, 1, 2, 2, 1], dtype=torch.int32)
    for u in (0.0, 0.3, 0.9999):
        w["uniform"][:] = u
        _check(drafts, w)


@pytest.mark.parametrize("sampled", [False, True])
def test_verify_tokens_outside(drafts, sampled):
    """Drafted tokens outside the vocabulary are rejected; parents that are none are followed by no one."""
    w = _world(14, [5, 5, 5], 40, "chain", sampled, keep=0.0)
    w["tokens"][2], w["tokens"][6], w["tokens"][11] = 40, -1, 1 << 30
    w["parents"][13] = 4
    w["parents"][14] = -7
    _check(drafts, w)


def test_verify_extremes(drafts):
    """Probabilities of 0 and 1: all kept, none kept, a residual of nothing, rows without a distribution."""
    V, n = 6, 4
    target = torch.zeros((3 * n + 3, V))
    target[:, 2] = 1
    draft = torch.zeros_like(target)
    draft[:, 2] = 1
    draft[n: 2 * n, 2], draft[n: 2 * n, 3] = 0, 1
    w = dict(tokens=torch.tensor([2] * n + [3] * n + [2] * n + [1, 1, 1], dtype=torch.int32),
             parents=torch.tensor(list(range(-1, n - 1)) * 3 + [-1, -1, -1], dtype=torch.int32),
             cu=torch.tensor([0, n, 2 * n, 3 * n, 3 * n + 1, 3 * n + 2, 3 * n + 3]).int(), target=target, draft=draft,
             uniform=torch.full((3 * n + 3,), 0.999), last=torch.tensor([0.0, 0.5, 0.9999999, 0.3, 0.3, 0.3]))
    target[2 * n, 2], target[2 * n, 0] = 0, 1            # kept token 2 has probability 0: rejected, the residual is token 0
    target[3 * n] = 0                                    # no distribution
    target[3 * n + 1] = float("nan")
    target[3 * n + 2, 4] = float("inf")
    assert _check(drafts, w) == [4, 1, 1, 1, 1, 1]
    w["draft"] = None
    _check(drafts, w)
    # the draft is the target and the token is rejected all the same (u draws 1): nothing is left, the target's row decides
    w = dict(tokens=torch.tensor([0, 1], dtype=torch.int32), parents=torch.tensor([-1, 0], dtype=torch.int32), cu=torch.tensor([0, 2]).int(),
             target=torch.tensor([[0.25, 0.25, 0.5], [1.0, 0, 0]]), uniform=torch.tensor([0.0, 1.0]), last=torch.tensor([0.6]))
    w["draft"] = w["target"].clone()
    assert _check(drafts, w) == [1]


def test_verify_last_borders(drafts):
    """Random numbers 0 and just below 1 draw the first and the last token that has a probability."""
    V = 9001
    w = _world(15, [1, 1, 1, 1], V, "chain", False)
    w["target"][:, : 4500] = 0
    w["target"][:, 8800:] = 0
    w["last"][:] = torch.tensor([0.0, 1 - 2.0 ** -24, 0.5, 2.0 ** -24])
    _check(drafts, w)
    out = _run(drafts, _cuda(w), 1)[2].flatten().tolist()
    assert out[0] == 4500 and out[1] == 8799


def test_verify_strides_and_rows_beyond(drafts):
    """Rows inside a larger tensor; tokens of no request are not looked at; a request larger than max_new is left out."""
    w = _world(16, [4, 9, 3], 100, "tree", True)
    g = _cuda(w)
    for n in ("target", "draft"):
        big = torch.full((20, 131), float("nan"), device="cuda")
        big[:16, 7:107] = g[n]
        g[n] = big[:, 7:107]
    for n, fill in (("tokens", 5), ("parents", 0), ("uniform", 0)):
        g[n] = torch.cat([g[n], torch.full((4,), fill, dtype=g[n].dtype, device="cuda")])
    path, counts, tokens = _run(drafts, g, 9)
    p, c, t = _expect(w, 9)
    assert counts.tolist() == c and path.tolist() == p and tokens.tolist() == t
    path, counts, tokens = _run(drafts, g, 5)
    p, c, t = [[r[:5] if n < 2 else r[:5] for r in x] for n, x in enumerate((p, [[n] for n in c], t))]
    for r in (0, 2):
        assert counts[r].item() == c[r][0] and path[r].tolist() == p[r] and tokens[r].tolist() == t[r]
    assert counts[1] == 0 and (path[1] == -1).all() and (tokens[1] == -1).all()


def test_verify_distribution(drafts):
    """Over many draws a step's first token follows the target's distribution, whatever
    drafted it.  20000 draws of 4 tokens: a frequency's standard deviation is at most
    0.0036; 5 of them are allowed."""
    R, V = 20000, 4
    g = torch.Generator().manual_seed(5)
    p, q = torch.tensor([0.1, 0.5, 0.25, 0.15]), torch.tensor([0.4, 0.1, 0.3, 0.2])
    drawn = torch.multinomial(q, 2 * R, replacement=True, generator=g).view(R, 2)
    for sampled in (True, False):
        kids = drawn if sampled else torch.tensor([[0, 2]]).expand(R, 2)
        tokens = torch.cat([torch.zeros((R, 1), dtype=torch.long), kids], 1).flatten().int()
        w = dict(tokens=tokens, parents=torch.tensor([-1, 0, 0], dtype=torch.int32).repeat(R), cu=torch.arange(0, 3 * R + 1, 3).int(),
                 target=p.expand(3 * R, V).contiguous(), draft=q.expand(3 * R, V).contiguous() if sampled else None,
                 uniform=torch.rand(3 * R, generator=g), last=torch.rand(R, generator=g))
        out = _run(drafts, _cuda(w), 3)[2][:, 0].cpu()
        freq = torch.bincount(out.long(), minlength=V).double() / R
        assert (freq - p.double()).abs().max() <= 5 * 0.0036


@pytest.mark.parametrize("sampled", [False, True])
def test_verify_streams_and_graph(drafts, sampled):
    w = _cuda(_world(17, [8, 5, 12], 5000, "tree", sampled))
    ref = [t.clone() for t in _run(drafts, w, 12)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    other = _run(drafts, w, 12, stream=side.cuda_stream)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, other))
    ws = torch.empty(drafts.verify_workspace(3, 5000), dtype=torch.uint8, device="cuda")
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        out = _run(drafts, w, 12, workspace=ws)
    for _ in range(3):
        ws.fill_(255)
        for t in out:
            t.fill_(7)
        _run(drafts, dict(w, uniform=w["uniform"] * 0.1), 12, workspace=ws)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(ref, out))


def test_verify_many_requests(drafts):
    _check(drafts, _world(18, [3, 1, 4] * 200, 30, "tree", True))


def test_refusals(drafts):
    from paper_2509_25689_amd import moeq
    w = _cuda(_world(19, [4, 2], 30, "tree", True))
    for name, bad in (("tokens", w["tokens"][:5]), ("tokens", w["tokens"].long()), ("parents", w["parents"][1:]), ("cu", w["cu"].long()),
                      ("target", w["target"].half()), ("target", w["target"][0]), ("draft", w["draft"][:, :29]), ("draft", w["draft"].double()),
                      ("uniform", w["uniform"][:3]), ("last", w["last"][:1]), ("last", w["last"].double()), ("target", w["target"].t().contiguous().t())):
        with pytest.raises(ValueError):
            _run(drafts, {**w, name: bad}, 4)
    with pytest.raises(TypeError):
        _run(drafts, {**w, "target": w["target"].cpu()}, 4)
    with pytest.raises(ValueError, match="gradient"):
        _run(drafts, {**w, "target": w["target"].clone().requires_grad_()}, 4)
    with pytest.raises(ValueError):
        _run(drafts, w, -1)
    with pytest.raises(moeq.MoeqError):
        _run(drafts, w, 257)
    with pytest.raises(moeq.MoeqError) as e:
        _run(drafts, w, 4, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == moeq.MOEQ_ERR_CAPACITY
    none = {**w, "tokens": w["tokens"][:0], "parents": w["parents"][:0], "cu": w["cu"][:1] * 0, "target": w["target"][:0],
            "draft": w["draft"][:0], "uniform": w["uniform"][:0], "last": w["last"][:0]}
    assert [t.shape for t in _run(drafts, none, 4)] == [(0, 4), (0,), (0, 4)]
