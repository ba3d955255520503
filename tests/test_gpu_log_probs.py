"""Log probabilities, entropy and top alternatives against the oracle in 64 bits (GPU).

Tolerance, with z = scale * logits, d = z - max z, u = 2^-24, E1 = sum p |d| and E2 = sum p d^2: a term exp(d) is off by 3 u |d| (difference, factor
and product) and 4 u of itself, the sum of them by u for each of a lane's n = vocab / 64 additions, at most, and 4 u for each of 30 joins: the
logarithm of the sum by L = u (3 E1 + n + 128) and 2 u of itself. lse adds the product scale * max and a sum: 4 u (|lse| + |max z|); a log probability
3 u |d_t| + 4 u (|log p| + |d_t|). Entropy: the weighted sum's terms by (3 u |d| + 8 u) |d| each and its additions alike: 3 u E2 + u (n + 136) E1,
and the logarithm's error, L (1 + E1)."""
from __future__ import annotations

import numpy as np
import pytest
import torch

from oracle import decode

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import U, gen, values  # noqa: E402

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


def run(z, targets=None, top=0, scale=1.0, **kw):
    rows, dev = z.shape[0], z.device
    out = dict(lse=torch.empty((rows,), device=dev), entropy=torch.empty((rows,), device=dev))
    if top:
        out.update(top_ids=torch.full((rows, top), -7, device=dev), top_logprobs=torch.empty((rows, top), device=dev))
    lp = None if targets is None else torch.empty(targets.shape, device=dev)
    A.log_probs(z, targets, lp, scale=scale, **out, **kw)
    return dict(out, lp=lp)


def check(z, targets, got, scale=1.0):
    zv, vocab = values(z) * np.float64(np.float32(scale)), z.shape[1]
    n = vocab / 64
    for i in range(z.shape[0]):
        lp, lse, h = decode.log_probs(zv[i])
        g = {k: None if v is None else v[i].cpu().numpy().astype(np.float64 if v.dtype == F32 else np.int64) for k, v in got.items()}
        if not np.isfinite(lse):
            same = lambda a, b: np.array_equal(np.asarray(a, dtype=np.float64), np.asarray(b, dtype=np.float64), equal_nan=True)  # noqa: E731
            assert same(g["lse"], lse) and same(g["entropy"], h)
        else:
            p, top = np.exp(lp), zv[i].max()
            d = np.where(p > 0, lp - lp.max(), 0.0)
            e1, e2 = (p * np.abs(d)).sum(), (p * d * d).sum()
            L = U * (3 * e1 + n + 128) + 2 * U * abs(lp.max())
            tol = lambda v: L + 7 * U * np.abs(v - lp.max()) + 4 * U * np.abs(v)  # noqa: E731
            assert abs(g["lse"] - lse) <= L + 4 * U * (abs(lse) + abs(top))
            assert abs(g["entropy"] - h) <= L * (1 + e1) + 3 * U * e2 + U * (n + 136) * e1 + 4 * U * h
        def near(a, ids):
            w = np.where(lp[ids] < -(2.0 ** 128 - 2.0 ** 103), -INF, lp[ids])      # rounds to -infinity in binary32
            if not np.isfinite(lse):
                assert np.array_equal(a, w, equal_nan=True)
                return
            fin = np.isfinite(w)
            assert np.array_equal(a[~fin], w[~fin]) and np.all(np.abs(a[fin] - w[fin]) <= tol(w[fin]))
        if targets is not None:
            t, a = targets[i].cpu().numpy().reshape(-1), g["lp"].reshape(-1)
            assert np.all(a[t < 0] == 0) and np.isnan(a[t >= vocab]).all()
            ok = (t >= 0) & (t < vocab)
            near(a[ok], t[ok])
        if got.get("top_ids") is not None:
            ids = g["top_ids"]
            if np.isnan(lse):
                assert (ids == -1).all() and np.isnan(g["top_logprobs"]).all()
            else:
                want = np.argsort(-values(z)[i], kind="stable")[:len(ids)]
                assert np.array_equal(ids, want)
                near(g["top_logprobs"], want)


def logits(g, rows, vocab, dtype, std=2.5):
    z = (torch.randn((rows, vocab), generator=g, device="cuda") * std).to(dtype)
    z[:, vocab // 3] += 9.0
    return z


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,vocab,top,scale", [
    (1, 1, 1, 1.0), (1, 7, 7, 0.5), (3, 64, 64, 1.0), (2, 255, 20, 1.3), (5, 2048, 64, 1.0), (4, 2049, 5, 1.0), (1, 8192, 20, 1.0), (2, 8191, 1, 2.0),
    (1, 32000, 5, 1.0), (3, 50001, 33, 0.7), (1, 131072, 64, 1.0), (70, 4097, 10, 1.0), (1200, 513, 3, 1.0), (1100, 2500, 0, 1.0), (1030, 9001, 17, 1.0),
    (2, 600011, 20, 1.0)])
def test_log_probs(rows, vocab, top, scale, dtype):
    g = gen(rows + vocab)
    z = logits(g, rows, vocab, dtype)
    t = torch.randint(0, vocab, (rows, 3), generator=g, device="cuda")
    t[0, 0] = 0
    t[-1, 1] = vocab - 1
    t[0, 2] = -100
    got = run(z, t, top, scale)
    some = torch.randperm(rows, generator=g, device="cuda")[:40]
    some = torch.cat((some, torch.tensor([0, rows - 1], device="cuda")))
    check(z[some], t[some], {k: None if v is None else v[some] for k, v in got.items()}, scale)
    if dtype != F32 or not top:
        return
    # each output alone gives the same
    for name in ("lse", "entropy"):
        only = torch.empty((rows,), device="cuda")
        A.log_probs(z, **{name: only}, scale=scale)
        # without the top values a row may be cut into the same chunks only
        assert torch.equal(only, got[name])
    ids = torch.empty((rows, top), dtype=torch.int64, device="cuda")
    A.log_probs(z, top_ids=ids, scale=scale)
    assert torch.equal(ids, got["top_ids"])
    lp = torch.empty((rows,), device="cuda")
    A.log_probs(z, t[:, 1].contiguous(), lp, scale=scale)
    assert torch.equal(lp, got["lp"][:, 1])


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,vocab", [(2, 40000), (1, 300), (1030, 3001)])
def test_masked_rows(rows, vocab, dtype):
    """-infinity nearly everywhere: fewer values than the top ones asked for, none at all, one at either end."""
    g = gen(vocab)
    z = logits(g, rows, vocab, dtype)
    for i, keep in enumerate(([5, vocab - 1], [0], [vocab - 1], [], list(range(40, 300, 7)), [vocab // 2])):
        r = (i * 37) % rows if rows > 6 else i % rows
        row = torch.full((vocab,), -INF, device="cuda", dtype=dtype)
        row[keep] = z[r, keep]
        one = z.clone()
        one[r] = row
        t = torch.tensor([keep[0] if keep else 3, vocab // 2, -1, vocab], device="cuda").repeat(rows, 1)
        got = run(one, t, 32)
        s = slice(r, r + 1)
        check(one[s], t[s], {k: v[s] for k, v in got.items()})


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", [700, 30000])
def test_equal_values(vocab, dtype):
    """All equal, all the type's lowest value but two, few different ones, zeros of both signs, ascending and descending
    rows: ties to the lowest token."""
    g = gen(vocab)
    low = torch.finfo(dtype).min
    rows = [torch.full((vocab,), 1.5), torch.full((vocab,), low), torch.randint(0, 3, (vocab,), generator=torch.Generator().manual_seed(1)).float(),
            torch.zeros(vocab) * (1 - 2 * (torch.arange(vocab) % 2)), torch.arange(vocab) / 100.0, -torch.arange(vocab) / 100.0,
            torch.full((vocab,), -0.0)]
    rows[1][[17, vocab - 2]] = torch.tensor([3.0, 4.0])
    z = torch.stack(rows).to("cuda").to(dtype)
    z[3] = torch.where(torch.arange(vocab, device="cuda") % 2 == 0, 0.0, -0.0).to(dtype)
    for top in (1, 20, 64):
        check(z, None, run(z, None, top))
    many = z[[0, 1, 2, 4] * 300]
    got = run(many, None, 20)
    check(many[-4:], None, {k: None if v is None else v[-4:] for k, v in got.items()})


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("vocab", [90, 20000])
def test_rows_that_are_not_finite(vocab, dtype):
    g = gen(3)
    z = logits(g, 5, vocab, dtype)
    clean = run(z, z.argmax(1, keepdim=True), 8)
    z[1, vocab - 1], z[3, 4] = NAN, INF
    t = torch.zeros((5, 2), dtype=torch.int64, device="cuda")
    t[:, 1] = -1
    got = run(z, t, 8)
    check(z, t, got)
    for i in (0, 2, 4):
        assert torch.equal(got["lse"][i], clean["lse"][i]) and torch.equal(got["top_ids"][i], clean["top_ids"][i])


def test_extreme_sizes():
    """Values as far apart as the type allows; scales near both ends."""
    z = torch.tensor([[3e38, -3e38, 1.0, 3e38], [1e-38, 0.0, -1e-38, 2e-38]], device="cuda")
    check(z, None, run(z, None, 4))
    with pytest.raises(A.AqmbError):               # differences that overflow would still weigh something
        run(z, None, 4, scale=1e-38)
    check(z, None, run(z, None, 4, scale=2.0 ** -120), scale=2.0 ** -120)
    check(z[1:], None, run(z[1:], None, 4, scale=1e38), scale=1e38)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_strided_rows_and_a_given_workspace(dtype):
    g = gen(5)
    wide = logits(g, 6, 70001, dtype)
    z = wide[::2, 3:66666]
    t = torch.randint(0, z.shape[1], (3, 2), generator=g, device="cuda")
    n = A.log_probs_workspace_bytes(dtype, 3, z.shape[1], 9)
    ws = torch.full((n + 64,), 255, dtype=torch.uint8, device="cuda")
    got = run(z, t, 9, workspace=ws[:n])
    check(z, t, got)
    assert (ws[n:] == 255).all()
    for a, b in zip(run(z, t, 9).values(), got.values()):
        assert torch.equal(a, b)


def test_a_row_does_not_depend_on_the_others():
    g = gen(8)
    z = logits(g, 9, 33000, BF16)
    a = run(z, None, 12)
    order = torch.randperm(9, generator=g, device="cuda")
    b = run(z[order], None, 12)
    for k in ("lse", "entropy", "top_ids", "top_logprobs"):
        assert torch.equal(a[k][order], b[k])


def test_refusals_of_the_binding():
    z = torch.zeros((2, 30), device="cuda")
    t, lp, f = torch.zeros((2, 1), dtype=torch.int64, device="cuda"), torch.zeros((2, 1), device="cuda"), torch.zeros((2,), device="cuda")
    for call in (lambda: A.log_probs(z), lambda: A.log_probs(z, t), lambda: A.log_probs(z, None, lp), lambda: A.log_probs(z, t.int(), lp),
                 lambda: A.log_probs(z, t, lp.double()), lambda: A.log_probs(z, t, f[:1]), lambda: A.log_probs(z[0], lse=f), lambda: A.log_probs(z.double(), lse=f),
                 lambda: A.log_probs(z, lse=f[:1]), lambda: A.log_probs(z, lse=f.half()), lambda: A.log_probs(z, entropy=f.cpu()), lambda: A.log_probs(z, lse=f, scale=0.0),
                 lambda: A.log_probs(z, top_ids=t.int()), lambda: A.log_probs(z, top_ids=t, top_logprobs=torch.zeros((2, 2), device="cuda")),
                 lambda: A.log_probs(z, top_ids=torch.zeros((2, 31), dtype=torch.int64, device="cuda")), lambda: A.log_probs(z[:0], lse=f[:0]),
                 lambda: A.log_probs(z.t(), lse=torch.zeros((30,), device="cuda")), lambda: A.log_probs(z[:, :0], lse=f),
                 lambda: A.log_probs(z.expand(2, 30)[:1].expand(2, 30), lse=f), lambda: A.log_probs(z, t.expand(2, 2), torch.zeros((2, 2), device="cuda"))):
        with pytest.raises(A.AqmbError):
            call()
