"""Draws of hs_sample at the borders between two logits, where the least
difference of two sums shows: the same token and count however many draws there
are."""
import numpy as np
import pytest
import torch

import pages_testutil as ref
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu


def at_borders(rows, V, k, T, borders, dtype, seed):
    """Rows of logits, and for each of them and of the first borders between two of its first k
    logits the fp32 number that is nearest to the share of the weights before it."""
    l = (torch.randn((rows, V), generator=ref.gen(seed), device="cuda") * 2.2).to(ref.DTYPES[dtype])
    z = l.double().topk(k, dim=1).values
    c = torch.exp((z - z[:, :1]) / T).cumsum(1)
    share = (c[:, :borders] / c[:, -1:]).to(torch.float32).flatten()
    return l, share, torch.arange(rows, device="cuda").repeat_interleave(borders).to(torch.int32)


def parts(l, n, by, **kw):
    """Tokens and counts, `by` draws a call."""
    got = [hs.hs_sample(l, **{name: x[i:i + by].contiguous() for name, x in kw.items()})
           for i in range(0, n, by)]
    return [torch.cat([g[j] for g in got]) for j in (0, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("what", ["u", "top_p"])
def test_the_same_however_many_draws(what, dtype):
    rows, V, k, borders = 1000, 9000, 400, 120
    n, differ = rows * borders, 0
    for seed, T in enumerate([0.7, 1.0, 1.3, 1.7, 2.0, 2.5, 3.0, 4.0]):
        l, share, row_of = at_borders(rows, V, k, T, borders, dtype, seed)
        kw = dict(temperature=torch.full((n,), T, device="cuda"), row_of=row_of,
                  top_k=torch.full((n,), k, **ref.INT), u=torch.full((n,), 0.5, device="cuda"))
        kw[what] = share.clamp(max=1 - 2.0 ** -24)
        many, some, few = (parts(l, m, by, **{x: y[:m] for x, y in kw.items()})
                           for m, by in ((n, n), (n, 300), (999, 3)))
        differ += sum((a != b).sum().item() for a, b in zip(many, some))
        differ += sum((a[:999] != b).sum().item() for a, b in zip(many, few))
    hs.hs_get_device_error()
    assert differ == 0


@pytest.mark.parametrize("V", [9000, 40000])
def test_the_same_of_rows_that_nothing_filters(V):
    """Sums of whole rows, of which 200 logits have nearly all."""
    rows, borders = 300, 30
    n, differ = rows * borders, 0
    for seed in range(4):
        l, _, row_of = at_borders(rows, V, 30, 1.0, borders, "bf16", 10 + seed)
        l[:, :200] += 8.0
        c = torch.exp(l.double().sort(1, descending=True).values - l.double().amax(1, True)).cumsum(1)
        u = (c[:, :borders] / c[:, -1:]).to(torch.float32).flatten().clamp(max=1 - 2.0 ** -24)
        many, some = (parts(l, n, by, u=u, row_of=row_of) for by in (n, 300))
        differ += sum((a != b).sum().item() for a, b in zip(many, some))
    hs.hs_get_device_error()
    assert differ == 0


@pytest.mark.parametrize("V", [3000, 9000])
def test_ends_and_equal_weights(V):
    """Shares that lie on a border exactly: none, of the first, of half of equal logits; and the
    largest number below 1."""
    n = 400
    l = torch.zeros((4, V), dtype=torch.bfloat16, device="cuda")
    l[1] = torch.randn(V, generator=ref.gen(1), device="cuda")
    l[2, :64] = 20.0
    l[3, 17] = 40.0
    row_of = (torch.arange(n, device="cuda") % 4).to(torch.int32)
    u = torch.tensor([0.0, 0.5, 0.25, 1 - 2.0 ** -24, 2.0 ** -24], device="cuda")[torch.arange(n, device="cuda") % 5]
    p = torch.tensor([1.0, 0.5, 0.0, 0.25, 1 - 2.0 ** -24, 0.75, 1.0], device="cuda")[
        torch.arange(n, device="cuda") % 7]
    k = torch.tensor([0, 1, 2, 64, 500, 2000], **ref.INT)[torch.arange(n, device="cuda") % 6]
    kw = dict(u=u, top_p=p, top_k=k, row_of=row_of)
    want = parts(l, n, n, **kw)
    for by in (1, 3, 100, 300):
        assert all(torch.equal(a, b) for a, b in zip(want, parts(l, n, by, **kw)))
    hs.hs_get_device_error()
    z = l.double().cpu().numpy()
    p32, u32 = p.double().tolist(), u.double().tolist()
    for i in range(n):
        token, _, count, sure = ref.sample(z[i % 4], 1.0, int(k[i]), p32[i], 0.0, u32[i])
        if sure:
            assert (want[0][i].item(), want[1][i].item()) == (token, count), i
