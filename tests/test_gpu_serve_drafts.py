"""Decode steps of a batch whose rows have different numbers of drafts: one
attention call per number of new tokens, one verification for all."""
import pytest
import torch

from tests import serve_ref as ref
from tests.test_gpu_serve import BF16, E4M3, F16, F32, Setup, drafted

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ds():
    from paper_2606_02982_amd import driftsched
    return driftsched


@pytest.mark.parametrize("qt,kt", [(BF16, BF16), (F16, F16), (BF16, E4M3)])
@pytest.mark.parametrize("window,sinks", [(0, 0), (64, 4)])
def test_rows_of_different_drafts(ds, qt, kt, window, sinks):
    """No request's weights are lost or counted twice: each query gives every
    head 1 in all, what older tokens had stays, what a rejected token had goes
    once its place is taken again."""
    n_req, batch, n_kv, group, dim, vocab, most, room = 14, 11, 2, 3, 64, 300, 4, 320
    g = torch.Generator().manual_seed(7)
    start = torch.randint(1, 250, (n_req,), generator=g).to(torch.int32)
    start[3], start[5] = 1, 64
    s = Setup(ds, start.tolist(), 16, n_kv, dim, kt, seed=8, width=room // 16)
    rows = torch.randperm(n_req, generator=g)[:batch].to(torch.int32)
    on_rows = rows.cuda()
    lens, mass = s.cache.lens, torch.rand((n_req, n_kv, room), generator=g).cuda()
    observed = torch.zeros(n_req, dtype=torch.int32, device="cuda")
    seen = 0
    for step in range(4):
        n_draft = torch.randint(0, most + 1, (batch,), generator=g).to(torch.int32)
        fresh = n_draft + 1                                   # the drafts and the token before them
        before = mass.clone()
        lens[on_rows.long()] += fresh.cuda()
        held = lens.cpu()
        for count in fresh.unique().tolist():
            part = rows[fresh == count]
            q = torch.randn((len(part), count, n_kv * group, dim), generator=g).to(qt)
            old = mass.cpu()
            out = ds.decode_attention(q.cuda(), s.cache, rows=part.cuda(), window=window, sinks=sinks, mass=mass, validate=True)
            want, off, m, m_off = ref.attention(q, s.k, s.v, s.table, held, part, window=window, sinks=sinks, mass=old,
                                                k_scale=s.scales[0], v_scale=s.scales[1])
            ref.check_out(out.cpu(), want, off, qt)
            ref.check_mass(mass.cpu(), m, m_off)
        for r, count in zip(rows.tolist(), fresh.tolist()):
            n = int(held[r])
            kept = before[r, :, :n - count].double().sum(-1)
            # weights of up to 320 tokens, each within 2^-15 of itself, and sums in 32 bits before
            given = mass[r, :, :n].double().sum(-1) - kept
            assert ((given - group * count).abs() <= 2.0 ** -12 * (group * count + kept)).all(), (step, r)
            assert (mass[r, :, n:] == before[r, :, n:]).all()
        p, qd, x, u, us, _ = drafted(batch, most, vocab, F32, 20 + step)
        out, emitted = ds.verify_draft(p.cuda(), qd.cuda(), x.cuda(), u.cuda(), us.cuda(), n_draft=n_draft.cuda(), rows=on_rows,
                                       observed=observed, lens=lens, validate=True)
        want = ref.verify(p, qd, x, u, us, n_draft)
        for i, (seq, a) in enumerate(want):
            assert out[i, :len(seq)].tolist() == seq and int(emitted[i]) == len(seq)
            assert int(lens[rows[i]]) == int(held[rows[i]]) - (int(n_draft[i]) - a)
        seen += int(emitted.sum())
    assert int(observed.sum()) == seen and int(lens.max()) <= room
