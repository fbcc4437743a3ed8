"""Key mass where query rows are unlike: rows that saw nothing over keys that hold anything, rows with
NaN or infinities, rows of very different size.  Against 64 bits."""
import pytest
import torch

from paper_2601_21927_gb300 import sonic
from tests.test_gpu_key_mass import check_mass, make
from tests.test_gpu_kv4 import dev, i32, status

pytestmark = pytest.mark.gpu
F = torch.float64


def spoil(K, bits, rows):
    """NaN in rows of the keys (in four bits: scale bytes that are NaN)."""
    if bits == 4:
        K[1][:, :, rows] = 255
    else:
        K[:, rows] = float("nan")


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("hq,hkv,d,queries,per_head", [(8, 2, 128, 1, True), (8, 2, 64, 3, True), (24, 2, 128, 1, False),
                                                       (28, 4, 128, 20, True), (16, 2, 64, 70, False)])
def test_rows_that_saw_nothing_over_any_keys(bits, hq, hkv, d, queries, per_head):
    """Sequences without a query, and with queries whose lse is -inf, keep keep * prev whatever their keys
    hold; beside them one whose first query alone saw nothing."""
    lens = [300, 260, 140, 150]
    K, K64, q, lse, start, rows, nq, q_start = make(hq, hkv, d, lens, queries, bits, 2, 5)
    nq[0] = 0
    gone = slice(q_start[1], q_start[1] + nq[1])
    q[:, gone], lse[:, gone] = float("nan"), -torch.inf
    for b in (0, 1):
        spoil(K, bits, slice(start[b], start[b] + lens[b]))
    if nq[3] > 1:
        q[:, q_start[3]], lse[:, q_start[3]] = float("inf"), -torch.inf
    before = torch.rand((2, hkv if per_head else 1, rows), device=dev())
    mass, prev, st = before.clone(), torch.rand_like(before), status()
    sonic.sonic_key_mass(q, K, lse, i32(lens), mass, kv_start=i32(start), max_len=300, q_start=i32(q_start),
                         q_len=i32(nq), max_q_len=queries, prev=prev, keep=0.5, status=st)
    assert st.item() == 0
    for b in (0, 1):
        sl = slice(start[b], start[b] + lens[b])
        assert torch.equal(mass[..., sl], 0.5 * prev[..., sl])
    K64, clean = K64.clone(), q.clone()
    for b in (0, 1):
        K64[:, start[b]:start[b] + lens[b]] = 0
    clean[:, gone] = 0
    if nq[3] > 1:
        clean[:, q_start[3]] = 0
    nq[0], lse[:, q_start[0]] = 1, -torch.inf  # (for the check: a row that saw nothing in the place of none)
    check_mass(mass, before, prev, 0.5, K64, clean, lse, start, lens, nq, q_start)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("hq,hkv,d,queries", [(8, 2, 128, 3), (28, 4, 128, 30), (16, 2, 64, 60)])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_a_bad_row_spoils_what_it_sees(bits, hq, hkv, d, queries, value):
    """One query row of one head holds NaN or an infinity (its lse as it comes): keys after it, and the
    other KV heads, have their exact sums."""
    lens = [400, 90]
    K, K64, q, lse, start, rows, nq, q_start = make(hq, hkv, d, lens, queries, bits, 1, 9)
    row, head = q_start[0] + 1, hq // hkv + 1  # a head of KV head 1
    sees = lens[0] - nq[0] + 2
    bad = q.clone()
    bad[:, row, head, 5] = value
    before = torch.rand((1, hkv, rows), device=dev())
    mass = before.clone()
    sonic.sonic_key_mass(bad, K, lse, i32(lens), mass, kv_start=i32(start), max_len=400, q_start=i32(q_start),
                         q_len=i32(nq), max_q_len=queries, keep=0.0)
    if value != value:
        assert bool(mass[0, 1, start[0]:start[0] + sees].isnan().all())
    # (what the row sees is filled in from a call without it)
    good = before.clone()
    sonic.sonic_key_mass(q, K, lse, i32(lens), good, kv_start=i32(start), max_len=400, q_start=i32(q_start),
                         q_len=i32(nq), max_q_len=queries, keep=0.0)
    mass[0, 1, start[0]:start[0] + sees] = good[0, 1, start[0]:start[0] + sees]
    check_mass(mass, before, None, 0.0, K64, q, lse, start, lens, nq, q_start)


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("hq,hkv,d,queries", [(28, 4, 128, 1), (28, 4, 128, 32), (16, 1, 64, 40), (4, 1, 128, 8)])
@pytest.mark.parametrize("power", [11, 12, 13, 20, 34, 60])
def test_rows_of_very_different_size(bits, hq, hkv, d, queries, power):
    """One head's queries are 2^power times the others', with an lse that leaves them no weight (they look at keys
    elsewhere); another head has one channel 2^10 times its others, which few keys answer.  Each row's
    scores are as exact as if it were alone.

    An element of a row is held in fp16 at a scale at which the row's largest lies at 2 or above: it is off by at most
    2^-25, 2^-26 of that largest, so a score by 2^-26 max|q| sum|k_d| scale, beside the 2^-21 of
    sum |q_d k_d| scale that check_mass derives."""
    lens = [500, 131]
    K, K64, q, lse, start, rows, nq, q_start = make(hq, hkv, d, lens, queries, bits, 1, 13)
    G = hq // hkv
    q = q.clone()
    q[:, :, 0] *= 2.0 ** power
    q[:, :, G - 1, 7] *= 2.0 ** 10
    scale, want = d ** -0.5, torch.zeros((1, hkv, rows), dtype=F, device=dev())
    tol = torch.full((1, hkv, rows), 1e-12, dtype=F, device=dev())
    inside = torch.zeros(rows, dtype=torch.bool, device=dev())
    terms = queries * G
    for b, n in enumerate(lens):
        sl = slice(start[b], start[b] + n)
        inside[sl] = True
        Kb = K64[0, sl].repeat_interleave(G, 1)
        for i in range(nq[b]):
            x = q[0, q_start[b] + i].to(F)
            S = torch.einsum("hd,thd->ht", x, Kb) * scale
            S[:, n - nq[b] + i + 1:] = -torch.inf
            z = torch.logsumexp(S, -1).float()
            z[0] = 2.0 * float(S[0, :n - nq[b] + i + 1].abs().max()) + 1000.0
            lse[0, q_start[b] + i] = z
            size = torch.einsum("hd,thd->ht", x.abs(), Kb.abs()) * scale
            reach = x.abs().amax(-1, keepdim=True) * Kb.abs().sum(-1).T * scale
            w = torch.exp(S - z[:, None].to(F))
            err = size * 2.0 ** -21 + reach * 2.0 ** -26 + 2.0 ** -19
            err[0] = 0
            want[0, :, sl] += w.view(hkv, G, n).sum(1)
            tol[0, :, sl] += (w * err).view(hkv, G, n).sum(1)
    tol += want * terms * 2.0 ** -23
    mass, st = torch.zeros((1, hkv, rows), device=dev()), status()
    sonic.sonic_key_mass(q, K, lse, i32(lens), mass, kv_start=i32(start), max_len=500, q_start=i32(q_start),
                         q_len=i32(nq), max_q_len=queries, keep=0.0, status=st)
    assert st.item() == 0
    bad = ~((mass.to(F) - want).abs() <= tol)
    assert not bool(bad[..., inside].any()), float(((mass.to(F) - want).abs() / tol)[..., inside].max())
