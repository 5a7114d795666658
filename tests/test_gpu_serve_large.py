"""The decode step at sizes where counters, chunks and offsets grow."""
import pytest
import torch

from tests import serve_ref as ref
from tests.test_gpu_serve import BF16, E4M3, F16, F32, Setup, ds, drafted, queries, run_evict, run_verify   # noqa: F401 (ds: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kt,t,group,window", [(BF16, 1, 20, 0), (E4M3, 2, 3, 0), (F16, 3, 12, 700001)])
def test_attention_of_a_million_tokens(ds, kt, t, group, window):   # noqa: F811
    n = 1000003
    s = Setup(ds, [n, 77], 64, 1, 16, kt, seed=1)
    s.attend(ds, queries(s, 2, t, group, 16, F16 if kt == F16 else BF16), window=window, mass=torch.rand((2, 1, n + 5), generator=s.g), max_len=n)


@pytest.mark.parametrize("n_kv,dim,kt", [(96, 64, BF16), (40, 16, E4M3), (33, 256, F16)])
def test_attention_of_many_heads(ds, n_kv, dim, kt):   # noqa: F811
    s = Setup(ds, [300, 1, 90], 16, n_kv, dim, kt, seed=n_kv)
    s.attend(ds, queries(s, 3, 2, 2 * n_kv, dim, BF16 if kt == E4M3 else kt), mass=torch.rand((3, n_kv, 304), generator=s.g))


def test_attention_of_far_tokens(ds):   # noqa: F811
    """Tokens of a page 2^27 elements apart: lane offsets that 32 bits do not hold."""
    step, page, dim = 1 << 27, 16, 64
    flat = torch.zeros(page * step, dtype=BF16, device="cuda")
    pool = flat.as_strided((3, page, 1, dim), (dim, step, 4 * dim, 1))
    g = torch.Generator().manual_seed(2)
    k = torch.randn((3, page, 1, dim), generator=g).to(BF16)
    for i in range(page):
        pool[:, i].copy_(k[:, i])
    table, lens = torch.tensor([[2, 0, 1]], dtype=torch.int32), torch.tensor([43], dtype=torch.int32)
    q = torch.randn((1, 2, 3, dim), generator=g).to(BF16)
    out = ds.decode_attention(q.cuda(), ds.kv_cache(pool, pool, table.cuda(), lens.cuda()), validate=True)
    want, off, _, _ = ref.attention(q, k, k, table, lens)
    ref.check_out(out.cpu(), want, off, BF16)
    del flat, pool


@pytest.mark.parametrize("inplace", [False, True])
def test_evict_of_two_million_tokens(ds, inplace):   # noqa: F811
    """More tokens than 256 chunks of 8,192."""
    n = (1 << 21) + 4001
    s = Setup(ds, [n, 30000], 64, 1, 16, E4M3, seed=2)
    r = torch.rand((2, 1, s.table.shape[1] * 64), generator=s.g)
    for mass in ((4 * r).exp(), (r * 3).floor()):
        run_evict(ds, s, torch.tensor([n * 0.4, 20000.5], dtype=torch.float64), mass, [1, 0], 4, 100, inplace=inplace)


@pytest.mark.parametrize("vocab,dtype", [((1 << 20) + 3, F16), (5000011, F32), (1 << 24, BF16)])
def test_verify_large_vocabularies(ds, vocab, dtype):   # noqa: F811
    p, q, x, u, us, g = drafted(3, 1, 1000, F32, 9)
    wide = torch.rand((3, 2, vocab), generator=g)
    wide = (wide / wide.sum(-1, keepdim=True)).to(dtype)
    other = torch.rand((3, 1, vocab), generator=g)
    other = (other / other.sum(-1, keepdim=True)).to(dtype)
    x = torch.randint(0, vocab, (3, 1), generator=g).to(torch.int32)
    run_verify(ds, wide, other, x, torch.tensor([[0.0], [0.999], [0.999]]), us)
    run_verify(ds, wide, None, x, torch.tensor([[0.0], [0.5], [0.5]]), torch.tensor([0.99999994, 0.99999994, 0.0]))
