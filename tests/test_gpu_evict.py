"""Eviction by attention weight on the GPU: rows, order and bytes exactly as the definition has
them, and the whole chain of a dialogue over a four-bit cache."""
import numpy as np
import pytest
import torch

from paper_2601_21927_gb300 import inputs, sonic
from tests import kv4_plain as plain
from tests.test_gpu_kv4 import check_decode, dev, empty4, i32, layout, random4, status

pytestmark = pytest.mark.gpu
BODY = sonic.ROLE_BODY


def expect(mass, role, keep_roles, recent, start, lens, budget):
    """Kept rows [layer][head][sequence] (absolute)."""
    out = []
    for m in mass.cpu().numpy():
        heads = []
        for h in m:
            seqs = []
            for s, n, k in zip(start, lens, budget):
                safe = [t >= n - recent or bool(role is not None and role[s + t] < 32 and keep_roles >> int(role[s + t]) & 1)
                        for t in range(n)]
                seqs.append([s + t for t in plain.evict_rows(h[s:s + n].tolist(), safe, k)])
            heads.append(seqs)
        out.append(heads)
    return out


def check(mass, parts_src, start, lens, budget, reserve=None, role=None, keep_roles=0, recent=0, spare=7,
          out_rows=None, give_src_idx=True, code=0, nl=None, hkv=None):
    ml, mh, rows = mass.shape
    want = expect(mass, role, keep_roles, recent, start, lens, budget)
    kept = [len(x) for x in want[0][0]]
    res = reserve or [0] * len(lens)
    offs = np.concatenate([[0], np.cumsum(np.array(kept, int) + res)]).astype(int)
    cap = int(offs[-1]) + spare if out_rows is None else out_rows
    dst = []
    for src in parts_src:
        shape = list(src.shape)
        shape[2 if src.dtype == torch.uint8 else 1] = cap
        dst.append(torch.full(shape, 3, dtype=src.dtype, device=dev()))
    offsets, out_len, st = i32([-1] * (len(lens) + 1)), i32([-1] * len(lens)), status()
    idx = torch.full((ml, mh, cap), -7, dtype=torch.int32, device=dev())
    omass = torch.full((ml, mh, cap), -7.0, device=dev())
    orole = torch.full((ml, mh, cap), 77, dtype=torch.uint8, device=dev())
    role_t = torch.from_numpy(role).to(dev()) if role is not None else None
    sonic.sonic_evict_kv(mass, list(zip(parts_src, dst)), i32(lens), offsets, kv_start=i32(start),
                         max_len=max(lens + [0]), budget=i32(budget), reserve=None if reserve is None else i32(reserve),
                         role=role_t, keep_roles=keep_roles, recent=recent, out_len=out_len,
                         src_idx=idx if give_src_idx else None, out_mass=omass,
                         out_role=orole if role is not None else None, status=st)
    assert st.item() == code
    assert offsets.tolist() == offs.tolist()
    assert out_len.tolist() == kept
    w_idx, w_mass, w_role = (x.cpu().clone().fill_(v) for x, v in ((idx, -7), (omass, -7.0), (orole, 77)))
    w_dst = [d.cpu().clone().fill_(3) for d in dst]
    for l in range(ml):
        for h in range(mh):
            for b, r in enumerate(want[l][h]):
                o = int(offs[b])
                n = min(len(r), max(0, cap - o))
                r = torch.tensor(r[:n], dtype=torch.long)
                w_idx[l, h, o:o + n] = r.int()
                w_idx[l, h, o + len(want[l][h][b]):int(offs[b + 1])] = -1
                w_role[l, h, o + len(want[l][h][b]):int(offs[b + 1])] = BODY
                w_mass[l, h, o:o + n] = mass.cpu()[l, h, r]
                if role is not None:
                    w_role[l, h, o:o + n] = torch.from_numpy(role)[r]
                for src, d in zip(parts_src, w_dst):
                    for ll in range(src.shape[0]) if ml == 1 else [l]:
                        heads = range(src.shape[1 if src.dtype == torch.uint8 else 2]) if mh == 1 else [h]
                        for hh in heads:
                            if src.dtype == torch.uint8:
                                d[ll, hh, o:o + n] = src.cpu()[ll, hh, r]
                            else:
                                d[ll, o:o + n, hh] = src.cpu()[ll, r, hh]
    if give_src_idx:
        assert torch.equal(idx.cpu(), w_idx)
    assert torch.equal(omass.cpu().nan_to_num(-99), w_mass.nan_to_num(-99))
    if role is not None:
        assert torch.equal(orole.cpu(), w_role)
    for g, w in zip(dst, w_dst):
        assert torch.equal(g.cpu().view(torch.uint8), w.view(torch.uint8))


def weights(ml, mh, rows, seed):
    """Attention weights as they come: over many magnitudes, with zeros and equal ones."""
    g = torch.Generator(device=dev())
    g.manual_seed(seed)
    m = torch.exp(4 * torch.randn((ml, mh, rows), generator=g, device=dev()))
    m[..., ::5] = 0
    m[..., 3::7] = 0.125
    return m


LENS = [[1], [0, 1, 2, 16, 33, 0], [700, 5, 2049, 64]]


@pytest.mark.parametrize("lens", LENS)
@pytest.mark.parametrize("per_layer,per_head", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("bits,hkv,d", [(16, 2, 128), (16, 1, 64), (4, 3, 64), (4, 2, 128)])
def test_evict(lens, per_layer, per_head, bits, hkv, d):
    nl = 3
    start, rows = layout(lens)
    rng = np.random.default_rng(len(lens) + hkv)
    role = rng.choice([0, 1, 2, 3], rows, p=[0.1, 0.2, 0.5, 0.2]).astype(np.uint8)
    if bits == 16:
        parts = [inputs.randn((nl, rows, hkv, d), k, device=dev()) for k in range(2)]
    else:
        parts = [*random4(nl, hkv, rows, d, 1), *random4(nl, hkv, rows, d, 2)]
    mass = weights(nl if per_layer else 1, hkv if per_head else 1, rows, 3)
    budget = [max(0, n // 2 - 1) for n in lens]
    check(mass, parts, start, lens, budget)
    check(mass, parts, start, lens, budget, reserve=[3 + b % 4 for b in range(len(lens))], role=role,
          keep_roles=1 << 0 | 1 << 3, recent=4, give_src_idx=False)


@pytest.mark.parametrize("budget", [[0, 0, 0], [1, 1, 1], [10_000, 300, 299], [299, 150, -5]])
def test_budgets_from_nothing_to_all(budget):
    lens = [300, 300, 300]
    start, rows = layout(lens)
    src = [inputs.randn((2, rows, 2, 64), 1, device=dev())]
    role = np.full(rows, 2, np.uint8)
    role[start[1]:start[1] + 40] = 0
    check(weights(2, 2, rows, 1), src, start, lens, budget, role=role, keep_roles=1, recent=0)
    check(weights(2, 2, rows, 1), src, start, lens, budget, role=role, keep_roles=1, recent=1000)


def test_order_of_special_masses():
    """NaN as -inf, -0 as 0, infinities, negative and denormal masses; ties to the lower row."""
    vals = [float("nan"), float("-inf"), float("inf"), 0.0, -0.0, 1e-45, -1e-45, 1.0, -1.0, 3.4e38, -3.4e38]
    rng = np.random.default_rng(0)
    m = torch.tensor(rng.choice(vals, (2, 2, 500)), dtype=torch.float32, device=dev())
    src = [inputs.randn((2, 500, 2, 64), 1, device=dev())]
    for k in range(0, 501, 25):
        check(m, src, [0], [500], [k])
    check(torch.zeros((1, 1, 500), device=dev()), src, [0], [500], [123])
    check(torch.full((1, 1, 500), float("nan"), device=dev()), src, [0], [500], [123])


@pytest.mark.parametrize("values", ["equal", "two", "near", "spread", "a few above"])
def test_keys_that_are_close_together(values):
    """Sequences of about as many rows as a block compares with one another, and longer ones of which as many
    are left: all equal, of two values, neighbours in the last bits, far apart, few of them large."""
    lens = [63, 64, 65, 128, 254, 255, 256, 257, 258, 513, 1025, 3000, 49_400 if values in ("near", "equal") else 700]
    start, rows = layout(lens)
    rng = np.random.default_rng(len(values))
    m = {"equal": np.full(rows, 0.75, np.float32),
         "two": rng.choice([0.75, 0.25], rows).astype(np.float32),
         "near": (0x3F400000 + rng.integers(0, 700, rows)).astype(np.int32).view(np.float32),
         "spread": np.exp(rng.uniform(-60, 60, rows)).astype(np.float32),
         "a few above": np.where(rng.random(rows) < 0.02, 5.0, rng.uniform(1, 1 + 2.0 ** -15, rows)).astype(np.float32)}
    mass = torch.from_numpy(m[values]).to(dev()).view(1, 1, rows)
    src = [inputs.randn((1, rows, 1, 64), 1, device=dev())]
    role = np.where(np.arange(rows) % 50 == 7, 0, 2).astype(np.uint8)
    for cut in (lambda n: 1, lambda n: n // 3, lambda n: n - 1, lambda n: n // 2 + 7):
        check(mass, src, start, lens, [cut(n) for n in lens])
        check(mass, src, start, lens, [cut(n) for n in lens], role=role, keep_roles=1, recent=3)


def test_long_sequences():
    """Longer than the keys that shared memory holds, beside short ones."""
    lens = [60_000, 49_152, 49_153, 10]
    start, rows = layout(lens)
    src = [inputs.randn((1, rows, 1, 64), 1, device=dev())]
    role = np.where(np.arange(rows) % 97 == 0, 0, 2).astype(np.uint8)
    check(weights(1, 1, rows, 2), src, start, lens, [20_001, 9000, 30_000, 5], role=role, keep_roles=1, recent=64)


def test_many_sequences():
    rng = np.random.default_rng(4)
    lens = rng.integers(0, 30, 1500).tolist()
    start, rows = layout(lens, gap=0)
    src = [random4(1, 1, rows, 64, 5)[1]]
    check(weights(1, 1, rows, 2), src, start, lens, [n // 3 for n in lens], reserve=[b % 3 for b in range(1500)])


@pytest.mark.parametrize("cap", [0, 1, 100, 160])
def test_capacity(cap):
    lens = [100, 90]
    start, rows = layout(lens)
    src = [inputs.randn((2, rows, 2, 64), 1, device=dev())]
    role = np.full(rows, 2, np.uint8)
    check(weights(2, 2, rows, 1), src, start, lens, [80, 70], reserve=[10, 5], role=role, out_rows=cap, code=4)


def test_piece_widths():
    """Arrays that start on 8 and on 4 bytes, and layers further apart than packed."""
    lens = [70, 33]
    start, rows = layout(lens)
    raw = torch.randint(0, 256, (2 * 3 * rows * 36 + 64,), dtype=torch.uint8, device=dev())
    for off in (0, 4, 8):
        src = raw[off:off + 2 * 3 * rows * 36].view(2, 3, rows, 36)
        check(weights(2, 3, rows, 1), [src], start, lens, [30, 20])
    wide = inputs.randn((2, rows + 9, 2, 64), 1, device=dev())[:, :rows]
    check(weights(2, 2, rows, 1), [wide], start, lens, [30, 20])


def test_refused_sequences_keep_nothing():
    rows = 100
    src = inputs.randn((1, rows, 1, 64), 1, device=dev())
    mass = weights(1, 1, rows, 1)
    for start, lens in (([0, 90], [20, 11]), ([0, -1], [20, 4]), ([0, 30], [20, 31]), ([0, 30], [20, -1])):
        dst, offsets, st = torch.zeros_like(src), i32([0] * 3), status()
        out_len = i32([9, 9])
        sonic.sonic_evict_kv(mass, [(src, dst)], i32(lens), offsets, kv_start=i32(start), max_len=30,
                             budget=i32([8, 8]), out_len=out_len, status=st)
        assert st.item() == 1 and offsets.tolist() == [0, 8, 8] and out_len.tolist() == [8, 0]
        assert bool((dst[:, 8:] == 0).all())


def test_without_parts_and_empty_batch():
    lens = [50, 20]
    start, rows = layout(lens)
    check(weights(2, 2, rows, 1), [], start, lens, [30, 20])
    off = i32([4])
    sonic.sonic_evict_kv(weights(1, 1, rows, 1), [], i32([]), off, kv_start=i32([]), max_len=0, budget=i32([]),
                         src_idx=torch.zeros((1, 1, 5), dtype=torch.int32, device=dev()))
    assert off.tolist() == [0]


def test_binding_refuses():
    src = inputs.randn((2, 40, 2, 64), 1, device=dev())
    mass = weights(2, 2, 40, 1)
    ok = dict(mass=mass, parts=[(src, torch.zeros_like(src))], lens=i32([40]), offsets=i32([0, 0]))
    kw = dict(kv_start=i32([0]), max_len=40, budget=i32([9]))
    other = torch.zeros((2, 40, 2, 32), dtype=torch.bfloat16, device=dev())
    for bad in (dict(mass=mass.double()), dict(mass=mass[..., :30]), dict(mass=weights(3, 2, 40, 1)),
                dict(parts=[(src, other)]), dict(parts=[(src.float(), src.float())]), dict(parts=[(src, src[:1])]),
                dict(parts=[(src, src)] * 5), dict(lens=i32([40, 1])), dict(offsets=i32([0])), dict(parts=[]),
                dict(budget=i32([1, 2])), dict(role=torch.zeros(39, dtype=torch.uint8, device=dev())),
                dict(keep_roles=1), dict(recent=-1), dict(src_idx=torch.zeros((2, 2, 39), dtype=torch.int32, device=dev()))):
        a, k = {**ok, **{x: v for x, v in bad.items() if x in ok}}, {**kw, **{x: v for x, v in bad.items() if x not in ok}}
        with pytest.raises(sonic.SonicError):
            sonic.sonic_evict_kv(*a.values(), **k)


def test_far_rows():
    """Attention weight and eviction where byte offsets pass 2^32 within one head's rows."""
    rows, d, n = 70_000_000, 128, 400
    start = [rows - n, 33_600_000]
    codes = torch.zeros((1, 1, rows, d // 2), dtype=torch.uint8, device=dev())
    scales = torch.zeros((1, 1, rows, d // 16), dtype=torch.uint8, device=dev())
    near = random4(1, 1, 2 * n, d, 9)
    for b, s in enumerate(start):
        codes[:, :, s:s + n], scales[:, :, s:s + n] = (x[:, :, b * n:(b + 1) * n] for x in near)
    q = inputs.randn((1, 2, 4, d), 1, device=dev()) * 0.3
    lse = torch.full((1, 2, 4), 3.0, device=dev())
    lens = i32([n, n])
    for max_q, kw in ((1, {}), (20, dict(q_start=i32([0, 1]), q_len=i32([1, 1])))):
        far, here = torch.zeros((1, 1, rows), device=dev()), torch.zeros((1, 1, 2 * n), device=dev())
        sonic.sonic_key_mass(q.to(torch.bfloat16), (codes, scales), lse, lens, far, kv_start=i32(start), max_len=n,
                             max_q_len=max_q, keep=0.0, **kw)
        sonic.sonic_key_mass(q.to(torch.bfloat16), near, lse, lens, here, kv_start=i32([0, n]), max_len=n,
                             max_q_len=max_q, keep=0.0, **kw)
        assert torch.equal(torch.cat([far[..., s:s + n] for s in start], -1), here)
    out = [[torch.zeros((1, 1, 300, x), dtype=torch.uint8, device=dev()) for x in (d // 2, d // 16)] for _ in range(2)]
    idx = [torch.zeros((1, 1, 300), dtype=torch.int32, device=dev()) for _ in range(2)]
    for k, (m, src, st) in enumerate(((far, (codes, scales), start), (here, near, [0, n]))):
        sonic.sonic_evict_kv(m, list(zip(src, out[k])), lens, i32([0, 0, 0]), kv_start=i32(st), max_len=n,
                             budget=i32([150, 150]), src_idx=idx[k])
    assert all(torch.equal(x, y) for x, y in zip(*out))
    assert torch.equal(idx[0][..., :150] - start[0], idx[1][..., :150])
    assert torch.equal(idx[0][..., 150:] - start[1], idx[1][..., 150:] - n)


def test_captured_and_on_another_stream():
    """Retention into four bits and an eviction of it in a graph, replayed on new weights, and both on a
    stream that is not the current one."""
    rng = np.random.default_rng(3)
    batch = inputs.Batch([inputs.random_dialogue(rng, max_body=90) for _ in range(5)])
    nl, hkv, d, T = 2, 2, 64, batch.total
    K, V = inputs.randn((nl, T, hkv, d), 1, device=dev()), inputs.randn((nl, T, hkv, d), 2, device=dev())
    role = torch.from_numpy(batch.role).to(dev())
    k_start, k_len = i32(batch.k_start), i32(batch.k_len)
    cap = sum(x.recipe_retained for x in batch.dialogues)

    def buffers():
        return dict(K4=empty4(nl, hkv, cap, d), V4=empty4(nl, hkv, cap, d), off=i32([0] * 6), n=i32([0] * 5),
                    mass=torch.zeros((nl, hkv, cap), device=dev()), out=i32([0] * 6),
                    idx=torch.zeros((nl, hkv, cap), dtype=torch.int32, device=dev()),
                    dst=[torch.zeros((nl, hkv, cap, x), dtype=torch.uint8, device=dev()) for x in (d // 2, d // 16) * 2])

    budget = i32([9, 3, 20, 0, 50])

    def both(b, ws, stream=None):
        w0 = sonic.sonic_kv4_compact(K, V, None, role, b["K4"], b["V4"], b["off"], k_start=k_start, k_len=k_len,
                                     ret_len=b["n"], workspace=ws[0], stream=stream)
        w1 = sonic.sonic_evict_kv(b["mass"], list(zip((*b["K4"], *b["V4"]), b["dst"])), b["n"], b["out"],
                                  kv_start=b["off"][:5], max_len=cap, budget=budget, src_idx=b["idx"], workspace=ws[1],
                                  stream=stream)
        return w0, w1

    b, side, e = buffers(), torch.cuda.Stream(), buffers()
    ws = both(b, (None, None))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(b, ws)
    for seed in (5, 6):
        b["mass"].copy_(weights(nl, hkv, cap, seed))
        e["mass"].copy_(b["mass"])
        torch.cuda.synchronize()
        g.replay()
        both(e, (None, None), side)
        torch.cuda.synchronize()
        off, n = b["off"].tolist(), b["n"].tolist()
        want = expect(b["mass"], None, 0, 0, off[:5], n, budget.tolist())
        at = b["out"].tolist()
        for l in range(nl):
            for h in range(hkv):
                for k in range(5):
                    assert b["idx"][l, h, at[k]:at[k + 1]].tolist() == want[l][h][k]
        for x, y in zip((*b["dst"], b["idx"], b["out"]), (*e["dst"], e["idx"], e["out"])):
            assert torch.equal(x, y)


def test_a_dialogue_in_four_bits():
    """Raw histories packed into a four-bit cache, a new turn prefilled over it, its rows stored,
    generation steps that collect attention weight, the cache brought down to a budget and a
    step over what is left: each step against 64 bits over what the cache holds."""
    nl, hq, hkv, d, B = 2, 8, 2, 128, 3
    batch = inputs.Batch([inputs.Dialogue(16, [(60, 12), (100, 20)], 0), inputs.Dialogue(5, [(30, 6)] * 7, 0),
                          inputs.Dialogue(40, [], 0)])
    T, turn = batch.total, 24
    K, V = inputs.randn((nl, T, hkv, d), 1, device=dev()), inputs.randn((nl, T, hkv, d), 2, device=dev())
    kept = [x.recipe_retained for x in batch.dialogues]
    cap = sum(kept) + B * (turn + 4)
    K4, V4, st = empty4(nl, hkv, cap, d), empty4(nl, hkv, cap, d), status()
    offsets, role = i32([0] * (B + 1)), torch.zeros(cap, dtype=torch.uint8, device=dev())
    seg = i32([0] * cap)
    sonic.sonic_kv4_compact(K, V, torch.from_numpy(batch.seg).to(dev()), torch.from_numpy(batch.role).to(dev()), K4, V4,
                            offsets, k_start=i32(batch.k_start), k_len=i32(batch.k_len), reserve=i32([turn + 4] * B),
                            out_role=role, out_seg=seg, status=st)
    start = offsets.tolist()[:B]
    # the new turn's keys and values go into the reserve rows, in four bits too
    tK, tV = inputs.randn((nl, B * turn, hkv, d), 3, device=dev()), inputs.randn((nl, B * turn, hkv, d), 4, device=dev())
    at = i32([start[b] + kept[b] + i for b in range(B) for i in range(turn)])
    sonic.sonic_kv4_store(tK, tV, K4, V4, dst_row=at, status=st)
    role[at.long()], seg[at.long()] = sonic.ROLE_CURR, 99
    wK, wV = torch.zeros((nl, cap, hkv, d), dtype=torch.bfloat16, device=dev()), torch.zeros(
        (nl, cap, hkv, d), dtype=torch.bfloat16, device=dev())
    sonic.sonic_kv4_load(K4, V4, wK, wV, status=st)
    assert torch.equal(wK.double(), plain.decode(*K4).transpose(1, 2))
    q = inputs.randn((nl, B * turn, hq, d), 5, device=dev())
    O, lse = torch.empty_like(q), torch.empty((nl, B * turn, hq), device=dev())
    lens = [n + turn for n in kept]
    sonic.sonic_attn_prefill(q, wK, wV, seg, role, O, k_start=i32(start), k_len=i32(lens),
                             q_start=i32([b * turn for b in range(B)]), q_len=i32([turn] * B), max_q_len=turn,
                             max_k_len=max(lens), lse=lse, status=st)
    # its queries' weight, and then that of three generation steps
    mass = torch.zeros((nl, hkv, cap), device=dev())
    sonic.sonic_key_mass(q, K4, lse, i32(lens), mass, kv_start=i32(start), max_len=max(lens),
                         q_start=i32([b * turn for b in range(B)]), q_len=i32([turn] * B), max_q_len=turn, status=st)
    for b in range(B):  # every query row gives its heads' weight of 1 each
        total = mass[:, :, start[b]:start[b] + lens[b]].double().sum((-1, -2))
        assert bool(((total - turn * hq).abs() < turn * hq * 1e-4).all())
    ws = None
    for s in range(3):
        nK, nV = (inputs.randn((nl, B, hkv, d), 20 + 2 * s + k, device=dev()) for k in range(2))
        sonic.sonic_kv4_store(nK, nV, K4, V4, dst_row=i32([start[b] + lens[b] for b in range(B)]), status=st)
        role[[start[b] + lens[b] for b in range(B)]] = sonic.ROLE_CURR
        lens = [n + 1 for n in lens]
        qs = inputs.randn((nl, B, hq, d), 40 + s, device=dev())
        Os, ls = torch.empty_like(qs), torch.empty((nl, B, hq), device=dev())
        ws = sonic.sonic_attn_decode_kv4(qs, K4, V4, i32(lens), Os, kv_start=i32(start), max_len=max(lens), lse=ls,
                                         status=st, workspace=ws)
        check_decode(Os, ls, qs, K4, V4, start, lens)
        before = mass.clone()
        sonic.sonic_key_mass(qs, K4, ls, i32(lens), mass, kv_start=i32(start), max_len=max(lens), prev=mass, status=st)
        gained = (mass - before).double()
        for b in range(B):
            assert bool(((gained[:, :, start[b]:start[b] + lens[b]].sum((-1, -2)) - hq).abs() < hq * 1e-3).all())
    assert st.item() == 0
    # down to 40 rows each, system rows and the last 8 kept whatever their weight
    dst = [torch.zeros((nl, hkv, B * 64, x), dtype=torch.uint8, device=dev()) for x in (d // 2, d // 16) * 2]
    offs, idx, out_len = i32([0] * (B + 1)), torch.zeros((nl, hkv, B * 64), dtype=torch.int32, device=dev()), i32([0] * B)
    src = [*K4, *V4]
    sonic.sonic_evict_kv(mass, list(zip(src, dst)), i32(lens), offs, kv_start=i32(start), max_len=max(lens),
                         budget=i32([40] * B), reserve=i32([4] * B), role=role, keep_roles=1 << sonic.ROLE_SYS,
                         recent=8, src_idx=idx, out_len=out_len, status=st)
    assert st.item() == 0
    want = expect(mass, role.cpu().numpy(), 1, 8, start, lens, [40] * B)
    new_start, new_lens = offs.tolist()[:B], out_len.tolist()
    assert new_lens == [40, 40, 48]
    for l in range(nl):
        for h in range(hkv):
            for b in range(B):
                assert idx[l, h, new_start[b]:new_start[b] + new_lens[b]].tolist() == want[l][h][b]
    qs = inputs.randn((nl, B, hq, d), 77, device=dev())
    Os = torch.empty_like(qs)
    sonic.sonic_attn_decode_kv4(qs, dst[:2], dst[2:], out_len, Os, kv_start=offs[:B].contiguous(), max_len=64, status=st)
    check_decode(Os, None, qs, dst[:2], dst[2:], new_start, new_lens)
    assert st.item() == 0


@pytest.mark.parametrize("bits", [4, 16])
def test_a_second_eviction(bits):
    """A cache whose heads chose for themselves is cut again by the weights that came out: system rows, a
    sequence's first, and the last ones lie in the same places in every head, so they stay again."""
    nl, hkv, d, lens = 2, 3, 64, [90, 400, 7]
    start, rows = layout(lens)
    role = np.full(rows, sonic.ROLE_NEXUS, np.uint8)
    for s in start:
        role[s:s + 6] = sonic.ROLE_SYS
    if bits == 4:
        src = [*random4(nl, hkv, rows, d, 3), *random4(nl, hkv, rows, d, 4)]
    else:
        src = [inputs.randn((nl, rows, hkv, d), k, device=dev()) for k in range(2)]
    cap = 200
    dst = [torch.zeros((nl, hkv, cap, x.shape[3]) if bits == 4 else (nl, cap, hkv, d), dtype=x.dtype, device=dev())
           for x in src]
    off, n, st = i32([0] * 4), i32([0] * 3), status()
    mass, role_t = weights(nl, hkv, rows, 9), torch.from_numpy(role).to(dev())
    omass = torch.zeros((nl, hkv, cap), device=dev())
    orole = torch.zeros((nl, hkv, cap), dtype=torch.uint8, device=dev())
    sonic.sonic_evict_kv(mass, list(zip(src, dst)), i32(lens), off, kv_start=i32(start), max_len=400,
                         budget=i32([40, 120, 30]), reserve=i32([8, 8, 8]), role=role_t, keep_roles=1 << sonic.ROLE_SYS,
                         recent=4, out_len=n, out_mass=omass, out_role=orole, status=st)
    assert st.item() == 0 and n.tolist() == [40, 120, 7] and off.tolist() == [0, 48, 176, 191]
    assert bool((orole == orole[:1, :1]).all())  # one list of roles serves every head
    check(omass, dst, off.tolist()[:3], n.tolist(), [25, 60, 2], reserve=[8, 0, 3], role=orole[0, 0].cpu().numpy(),
          keep_roles=1 << sonic.ROLE_SYS, recent=4)
