"""Log probabilities of many rows (GPU): texts without top values in 16 bits, and rows long and many enough for a wave each
with top values. Tolerances are those of test_gpu_log_probs.py."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2606_12876_amd as A  # noqa: E402
from ops_helpers import gen, normal  # noqa: E402
from test_gpu_log_probs import BF16, F16, F32, INF, NAN, check, logits, run  # noqa: E402


def part(got, rows):
    return {k: None if v is None else v[rows] for k, v in got.items()}


def sample(g, rows, *more, n=25):
    return torch.cat((torch.randperm(rows, generator=g, device="cuda")[:n], torch.tensor([0, rows - 1, *more], device="cuda")))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,vocab,scale", [(1100, 50001, 1.0), (1300, 33001, 0.7), (1024, 8200, 1.0), (2600, 16384, 1.3), (3, 300007, 1.0), (4200, 9000, 1.0)])
def test_a_text_without_top_values(rows, vocab, scale, dtype):
    g = gen(vocab)
    wide = normal(g, rows, vocab + 5, dtype=dtype, std=2.5)
    for z in (wide[:, 2:2 + vocab], wide[:, 2:2 + vocab].contiguous()):
        z[1].fill_(-INF)
        z[2 % rows, vocab // 2:] = -INF
        t = torch.randint(0, vocab, (rows, 2), generator=g, device="cuda")
        t[0, 0], t[1, 1], t[-1, 0] = vocab - 1, -1, 0
        got = run(z, t, 0, scale)
        s = sample(g, rows, 1, 2 % rows)
        check(z[s], t[s], part(got, s), scale)
        only = torch.empty((rows,), device="cuda")
        A.log_probs(z, lse=only, scale=scale)
        assert torch.equal(only, got["lse"])


@pytest.mark.parametrize("dtype,vocab", [(BF16, 32000), (F16, 9001), (F16, 32768), (F32, 4500), (F32, 16000), (BF16, 32769)])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_many_rows_with_top_values(top, dtype, vocab):
    """From 4096 rows on a wave takes a row by itself, up to 64 loads of it; 32769 values are one more."""
    rows = 4099
    g = gen(vocab + top)
    z = logits(g, rows, vocab, dtype)
    low = torch.finfo(dtype).min
    z[3].fill_(1.5)
    z[4].fill_(-INF)
    z[5].fill_(low)
    z[5, [17, vocab - 2]] = torch.tensor([3.0, 4.0], dtype=dtype, device="cuda")
    z[6, 4:] = -INF
    z[7] = (torch.arange(vocab, device="cuda") / vocab * 8).to(dtype)
    z[8] = -z[7]
    z[9] = torch.randint(0, 3, (vocab,), generator=g, device="cuda").to(dtype)
    z[10, vocab - 1], z[11, vocab // 2], z[12, 0] = NAN, INF, -INF
    t = torch.randint(0, vocab, (rows, 1), generator=g, device="cuda")
    got = run(z, t, top)
    s = sample(g, rows, *range(3, 13))
    check(z[s], t[s], part(got, s))
    want = torch.topk(z[13:].float(), top).values
    assert torch.equal(z[13:].gather(1, got["top_ids"][13:]).float(), want)                # all of them


@pytest.mark.parametrize("rows", [15, 16, 17])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_on_either_side_of_a_number_of_workgroups(rows, dtype):
    g = gen(rows)
    z = logits(g, rows, 131072, dtype)
    z.masked_fill_(torch.rand(z.shape, generator=g, device="cuda") < 0.5, -INF)
    t = torch.randint(0, 131072, (rows, 2), generator=g, device="cuda")
    check(z, t, run(z, t, 20, 1.25), 1.25)
