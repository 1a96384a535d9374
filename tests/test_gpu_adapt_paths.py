"""Ways of the adapters' calls that ordinary sizes do not take: ids out of range where the rows are put in order first, many adapters for few
rows, the last size whose workgroups find their tiles by themselves."""
import numpy as np
import pytest
import torch

import plain_block as P
from paper_2605_22428_amd import binding as B
from test_gpu_adapt import DEV, GAMMA, Set, close, mixed, normal

pytestmark = pytest.mark.gpu


def gradients(s, ids, flags):
    T = len(ids)
    x, dy, h = normal(5, T, s.n_in).bfloat16(), normal(6, T, s.n_out).bfloat16(), normal(8, T, s.rank)
    dx, da, db = torch.empty((T, s.n_in), dtype=torch.bfloat16, device=DEV), torch.empty_like(s.dev._held[0]), torch.empty_like(s.dev._held[1])
    ws = s.dev.workspace(T)
    ws.fill_(0xff)
    s.dev.mw_adapt_backward(x.to(DEV), torch.from_numpy(ids).to(DEV), h.to(DEV), dy.to(DEV), None, dx, da, db, ws, flags)
    torch.cuda.synchronize()
    want = P.adapt_backward(x.double().numpy(), ids, h.double().numpy(), dy.double().numpy(), np.zeros((T, s.n_in)), s.a, s.b, s.scale, GAMMA)
    for got, (v, off) in zip((dx, da, db), want):
        close(got.float().cpu().numpy(), v, off)


@pytest.mark.parametrize("T", [5, 256, 257, 300, 9000])
def test_ids_out_of_range(T):
    """In front, in the middle and at the end of the pieces that rows are looked at in."""
    s = Set(4, 16, 64, 64)
    x, base, ids = normal(5, T, 64).bfloat16(), normal(6, T, 64).bfloat16(), mixed(T, T, 4)
    for wrong in (False, True):
        if wrong:
            ids[[0, T // 2, T - 1]] = 4, -2, 2 ** 31 - 1
            ids[T // 3] = -2 ** 31
        for call in (lambda f: s.check(x, ids, base, flags=f), lambda f: gradients(s, ids, f)):
            flags = torch.zeros(1, dtype=torch.int32, device=DEV)
            call(flags)
            assert int(flags) == (B.MW_FLAG_BAD_ADAPTER if wrong else 0)


@pytest.mark.parametrize("T,n,rank,n_in,n_out", [(64, 1024, 8, 16, 16), (200, 300, 8, 64, 16), (256, 64, 16, 72, 40), (256, 1024, 16, 40, 24), (1, 1024, 8, 16, 16)])
def test_many_adapters_for_few_rows(T, n, rank, n_in, n_out):
    """Workgroups that find their tile in several turns over the adapters."""
    s = Set(n, rank, n_in, n_out)
    x, base = normal(5, T, n_in).bfloat16(), normal(6, T, n_out).bfloat16()
    for ids in (mixed(T, T, n), np.full(T, n - 1, dtype=np.int32), (np.arange(T) * 257 % n).astype(np.int32)):
        s.check(x, ids, base)
    gradients(s, mixed(T, T, n), None)
