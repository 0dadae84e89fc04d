"""KvRequests: prompts of several workflows, equal ones merged, through the
paged cache and its attention, against attention computed prompt by prompt
in 64 bits from the values that the cache's codes stand for."""
import numpy as np
import pytest
import torch

import kv_testutil as ref
import paper_2607_22578_gb300 as hs

pytestmark = pytest.mark.gpu
H, G, D, BT = 2, 4, 64, 16


def embed(tokens, pos, rows, seed):
    """Values of a token at a position: the same wherever the pair occurs."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = torch.randn((64, rows * D), generator=g, device="cuda")
    p = torch.randn((512, rows * D), generator=g, device="cuda")
    return (t[tokens.long()] + p[pos.long()]).view(-1, rows, D).to(torch.bfloat16)


def tokens_of(req, prompts, lens, step):
    """(token ids, positions) of the batch's merged tokens, in the order of their slots."""
    starts = req.starts.tolist()
    ids, pos = [], []
    for u in range(int(req.n_req.item())):
        p = torch.arange(lens[u] - (starts[u + 1] - starts[u]), lens[u])
        pos.append(p)
        ids.append(torch.tensor(prompts[u])[p] if step == 0 else torch.full((len(p),), step))
    return torch.cat(ids).cuda(), torch.cat(pos).cuda()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_merged_prompts_then_steps(fmt):
    rng = np.random.default_rng(3)
    base = [rng.integers(0, 64, size=n).tolist() for n in (40, 17, 100, 3)]
    which = [0, 1, 0, 2, 3, 1, 2, 0]                   # eight workflows, four different prompts
    stride = 100
    tokens = np.full((len(which), stride), 63)
    for i, w in enumerate(which):
        tokens[i, :len(base[w])] = base[w]
    lens = torch.tensor([len(base[w]) for w in which], dtype=torch.int32, device="cuda")
    cache = hs.KvCache(32, BT, H, D, ref.CODES[fmt])
    req = hs.KvRequests(cache, max_requests=10, max_len=160)
    slots, starts, unique_idx, inverse = req.begin(
        torch.from_numpy(tokens).int().cuda(), lens)
    assert int(req.n_req.item()) == 4 and inverse.tolist() == which
    assert unique_idx[:4].tolist() == [0, 1, 3, 4]
    have = [40, 17, 100, 3]
    assert req.lens.tolist() == have + [0] * 6 and starts.tolist()[:5] == [0, 40, 57, 157, 160]
    for step in range(3):
        if step:
            fresh = torch.zeros(10, dtype=torch.int32, device="cuda")
            fresh[:4] = 1
            req.extend(fresh, 10, 1)
            have = [x + 1 for x in have]
        ids, pos = tokens_of(req, base, have, step)
        n, T = len(ids), len(req.slots)
        assert (req.slots[:n] >= 0).all() and (req.slots[n:] == -1).all()
        q, k, v = (torch.zeros((T, r, D), dtype=torch.bfloat16, device="cuda") for r in (H * G, H, H))
        for i, x in enumerate((q, k, v)):
            x[:n] = embed(ids, pos, x.shape[1], i)
        req.append(cache, k, v)
        out, lse = req.attend(cache, q)
        hs.hs_get_device_error()
        want, _, tol, _ = ref.attend(q[:n], cache.k, cache.v, cache.k_scale, cache.v_scale, fmt,
                                     req.table, have, req.starts.tolist()[:5], D ** -0.5, True, 0)
        least, most = ((want + x).to(torch.bfloat16) for x in (-tol, tol))
        assert ((out[:n] >= least) & (out[:n] <= most)).all()
        # what the cache stands for is what was written, to half a step of its codes
        for c, s, x in ((cache.k, cache.k_scale, k), (cache.v, cache.v_scale, v)):
            at = req.slots[:n].long()
            code = torch.from_numpy(ref.values(ref.to_bytes(c), fmt)).cuda()
            got = code[at // BT, :, at % BT] * s.double()[at // BT][..., None]
            step_of = s.double()[at // BT][..., None] if fmt == "int8" else \
                torch.maximum(got.abs() / 8, s.double()[at // BT][..., None] * 2.0 ** -9)
            assert ((got - x[:n].double()).abs() <= 0.5 * step_of * (1 + 1e-12)).all()
    free = int((req.cursor[1] - req.cursor[0]).item())
    done = torch.zeros(10, dtype=torch.bool, device="cuda")
    done[2] = True
    req.release(done)
    hs.hs_get_device_error()
    assert int((req.cursor[1] - req.cursor[0]).item()) == free + 7 and req.lens.tolist()[2] == 0
