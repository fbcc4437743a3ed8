"""Four-bit caches on the GPU: packing and unpacking (exact), decode over them against 64 bits."""
import numpy as np
import pytest
import torch

from paper_2601_21927_gb300 import inputs, sonic
from tests import kv4_plain as plain

pytestmark = pytest.mark.gpu
F = torch.float64


def dev():
    return torch.device("cuda:0")


def i32(a):
    return torch.tensor(list(a), dtype=torch.int32, device=dev())


def status():
    return torch.zeros(1, dtype=torch.int32, device=dev())


def empty4(nl, hkv, rows, d, fill=0):
    return (torch.full((nl, hkv, rows, d // 2), fill, dtype=torch.uint8, device=dev()),
            torch.full((nl, hkv, rows, d // 16), fill, dtype=torch.uint8, device=dev()))


def random4(nl, hkv, rows, d, seed, lo=96, hi=130):
    """A cache of random codes and of scales around 1 (bytes lo .. hi - 1)."""
    g = torch.Generator(device=dev())
    g.manual_seed(seed)
    return (torch.randint(0, 256, (nl, hkv, rows, d // 2), generator=g, device=dev(), dtype=torch.uint8),
            torch.randint(lo, hi, (nl, hkv, rows, d // 16), generator=g, device=dev(), dtype=torch.uint8))


def special_rows(d):
    """bf16 rows that hold every border between two codes at many scales, borders of the scale
    grid, infinities, NaN, zeros, and the ends of the range."""
    rows = []
    for e in range(-20, 16):
        for m in (1.0, 1.125, 1.25, 1.375, 1.5, 1.625, 1.75, 1.875):
            s = m * 2.0 ** e
            blk = [6 * s] + [t * s for t in (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)]
            blk += [-b for b in blk]
            rows.append(blk)
    for top in (6.375, 0.0, 2.0 ** -16, 3 * 2.0 ** -17, 6 * 2.0 ** -18, 61440.0, 1e30, 3.3e38):
        rows.append([top, -top] + [top / k for k in range(1, 15)])
    inf, nan = float("inf"), float("nan")
    rows += [[inf] + [1.0] * 15, [-inf, nan] + [2.0] * 14, [nan] * 16, [nan, 1.0, -2.0] + [0.5] * 13,
             [-0.0] * 16]
    g = torch.Generator().manual_seed(5)
    rnd = torch.randn((200, 16), generator=g) * torch.exp(3 * torch.randn((200, 1), generator=g))
    t = torch.cat([torch.tensor(rows), rnd]).to(torch.bfloat16)
    n = t.shape[0] // (d // 16) * (d // 16)
    return t[:n].reshape(-1, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hkv", [1, 3, 8])
def test_store_and_load_are_exact(d, hkv):
    base = special_rows(d)
    n, nl = base.shape[0], 2
    K = torch.stack([torch.stack([base.roll(h + 3 * l, 0) for h in range(hkv)], 1) for l in range(nl)]).to(dev())
    V = K.flip(1).contiguous()
    K4, V4, st = empty4(nl, hkv, n, d, 77), empty4(nl, hkv, n, d, 77), status()
    sonic.sonic_kv4_store(K, V, K4, V4, status=st)
    oK, oV = torch.empty_like(K), torch.empty_like(V)
    sonic.sonic_kv4_load(K4, V4, oK, oV, status=st)
    assert st.item() == 0
    for X, X4, oX in ((K, K4, oK), (V, V4, oV)):
        codes, scales = plain.encode(X.transpose(1, 2))
        got = plain.decode(X4[0].cpu(), X4[1].cpu())
        assert torch.equal(X4[1].cpu(), scales)
        assert torch.equal(got, plain.decode(codes, scales))  # (values: -0 is 0)
        assert torch.equal(oX.cpu().double(), got.transpose(1, 2))


@pytest.mark.parametrize("d,hkv,n", [(128, 8, 1), (64, 1, 1), (64, 2, 333), (128, 4, 1025)])
def test_rows_by_index(d, hkv, n):
    """Source and destination lists, skipped rows (-1), rows out of range, a layer stride."""
    nl, T, rows = 3, n + 7, n + 40
    buf = inputs.randn((nl, T + 5, hkv, d), 3, device=dev())
    K, V = buf[:, :T], (buf * 0.5)[:, 5:]
    rng = np.random.default_rng(n)
    src, dst = rng.permutation(T)[:n], rng.permutation(rows)[:n]
    if n > 2:
        src[1] = -1
    K4, V4, st = empty4(nl, hkv, rows, d, 9), empty4(nl, hkv, rows, d, 9), status()
    sonic.sonic_kv4_store(K, V, K4, V4, src_row=i32(src), dst_row=i32(dst), status=st)
    assert st.item() == 0
    ok = src >= 0
    for X, X4 in ((K, K4), (V, V4)):
        want = [torch.full_like(X4[0].cpu(), 9), torch.full_like(X4[1].cpu(), 9)]
        codes, scales = plain.encode(X[:, src[ok]].transpose(1, 2))
        want[0][:, :, dst[ok]], want[1][:, :, dst[ok]] = codes, scales
        assert torch.equal(X4[1].cpu(), want[1])
        sel = np.setdiff1d(np.arange(rows), dst[ok])
        assert torch.equal(X4[0].cpu()[:, :, sel], want[0][:, :, sel])
        assert torch.equal(plain.decode(X4[0].cpu(), X4[1].cpu()), plain.decode(*want))
    # back: rows dst of the cache to rows src of new buffers
    oK, oV = torch.full_like(buf, 3.0)[:, :T], torch.full_like(buf, 3.0)[:, 2:T + 2]
    sonic.sonic_kv4_load(K4, V4, oK, oV, src_row=i32(np.where(ok, dst, -1)), dst_row=i32(np.maximum(src, 0)),
                         status=st)
    assert st.item() == 0
    for X4, oX in ((K4, oK), (V4, oV)):
        want = torch.full(oX.shape, 3.0, dtype=F)
        want[:, src[ok]] = plain.decode(X4[0].cpu(), X4[1].cpu())[:, :, dst[ok]].transpose(1, 2)
        assert torch.equal(oX.cpu().double(), want)


def test_free_rows_are_left_out():
    """A whole cache read with the compaction's src_idx: its free rows are not."""
    hkv, d = 2, 64
    K4, V4 = random4(2, hkv, 50, d, 1), random4(2, hkv, 50, d, 2)
    live = i32([-1 if j % 7 == 3 or j > 40 else 1000 + j for j in range(50)])
    oK, oV = (torch.full((2, 50, hkv, d), 5.0, dtype=torch.bfloat16, device=dev()) for _ in range(2))
    sonic.sonic_kv4_load(K4, V4, oK, oV, live=live)
    gone = live.cpu() < 0
    for X4, oX in ((K4, oK), (V4, oV)):
        want = plain.decode(*X4).cpu().transpose(1, 2)
        assert torch.equal(oX.cpu().double()[:, ~gone], want[:, ~gone])
        assert bool((oX.cpu()[:, gone] == 5).all())
    n4, m4 = empty4(2, hkv, 50, d, 3), empty4(2, hkv, 50, d, 3)
    sonic.sonic_kv4_store(oK, oV, n4, m4, live=live[:45].contiguous())
    assert bool((n4[0][:, :, 45:] == 3).all()) and bool((n4[0].cpu()[:, :, gone] == 3).all())
    want = plain.decode(*plain.encode(oK.transpose(1, 2)))  # (a block without a 6 is packed anew)
    assert torch.equal(plain.decode(*n4).cpu()[:, :, ~gone], want[:, :, ~gone])


def test_rows_out_of_range_are_skipped_and_told():
    d, hkv = 64, 2
    K = inputs.randn((1, 6, hkv, d), 1, device=dev())
    for src, dst, code in (([0, 6, 2], [0, 1, 2], 1), ([0, -2, 2], [0, 1, 2], 1), ([0, 1, 2], [0, 9, 2], 4),
                           ([0, 1, 2], [0, -1, 2], 4)):
        K4, V4, st = empty4(1, hkv, 9, d, 5), empty4(1, hkv, 9, d, 5), status()
        sonic.sonic_kv4_store(K, K, K4, V4, src_row=i32(src), dst_row=i32(dst), status=st)
        assert st.item() == code
        codes, scales = plain.encode(K[:, [0, 2]].transpose(1, 2))
        assert torch.equal(K4[1].cpu()[:, :, [0, 2]], scales)
        assert bool((K4[1].cpu()[:, :, [1, 3, 8]] == 5).all())
    # the cache is the source of a load: its rows are checked as such
    K4, V4 = random4(1, hkv, 4, d, 3), random4(1, hkv, 4, d, 4)
    for src, dst, code in (([0, 4], [0, 1], 1), ([0, 1], [0, 6], 4)):
        out, st = torch.full_like(K, 7.0), status()
        sonic.sonic_kv4_load(K4, V4, out, out.clone(), src_row=i32(src), dst_row=i32(dst), status=st)
        assert st.item() == code
        assert bool((out[:, 1:] == 7).all()) and not bool((out[:, 0] == 7).all())


@pytest.mark.parametrize("d,hkv", [(64, 1), (128, 4)])
def test_compact_into_four_bits(d, hkv):
    """The retention rule's rows, each packed: against sonic_compact_kv and the plain format."""
    rng = np.random.default_rng(7)
    batch = inputs.Batch([inputs.random_dialogue(rng) for _ in range(9)])
    nl, T = 2, batch.total
    K, V = inputs.randn((nl, T, hkv, d), 1, device=dev()), inputs.randn((nl, T, hkv, d), 2, device=dev())
    role, seg = torch.from_numpy(batch.role).to(dev()), torch.from_numpy(batch.seg).to(dev())
    keep = [x.recipe_retained for x in batch.dialogues]
    reserve = i32([3, 0, 5, 1, 0, 0, 2, 8, 4])
    need = sum(keep) + int(reserve.sum())
    for cap, code in ((need + 6, 0), (need - 11, 4)):
        res = {}
        for kind in ("bf16", "four"):
            r = dict(offsets=i32([0] * 10), ret_len=i32([0] * 9), src_idx=i32([-5] * cap),
                     out_role=torch.full((cap,), 99, dtype=torch.uint8, device=dev()), out_seg=i32([-9] * cap),
                     status=status())
            kw = dict(k_start=i32(batch.k_start), k_len=i32(batch.k_len), reserve=reserve,
                      **{k: r[k] for k in ("ret_len", "src_idx", "out_role", "out_seg", "status")})
            if kind == "bf16":
                o = [torch.zeros((nl, cap, hkv, d), dtype=torch.bfloat16, device=dev()) for _ in range(2)]
                sonic.sonic_compact_kv(K, V, seg, role, *o, r["offsets"], **kw)
            else:
                o = [empty4(nl, hkv, cap, d, 200), empty4(nl, hkv, cap, d, 200)]
                sonic.sonic_kv4_compact(K, V, seg, role, *o, r["offsets"], **kw)
            res[kind] = (r, o)
        for k in res["bf16"][0]:
            assert torch.equal(res["bf16"][0][k], res["four"][0][k]), k
        assert res["four"][0]["status"].item() == code
        off, lens = res["four"][0]["offsets"].tolist(), res["four"][0]["ret_len"].tolist()
        written = np.zeros(cap, bool)
        for b, n in enumerate(lens):
            written[off[b]:min(cap, off[b] + n)] = True
        for bf, four in zip(res["bf16"][1], res["four"][1]):
            codes, scales = plain.encode(bf.transpose(1, 2))
            assert torch.equal(four[1].cpu()[:, :, written], scales[:, :, written])
            assert torch.equal(plain.decode(four[0].cpu(), four[1].cpu().clamp(max=226))[:, :, written],
                               plain.decode(codes, scales)[:, :, written])
            assert bool((four[0].cpu()[:, :, ~written] == 200).all())
            assert bool((four[1].cpu()[:, :, ~written] == 200).all())


def test_compact_empty_batch_and_no_capacity():
    K = inputs.randn((1, 8, 1, 64), 1, device=dev())
    role = torch.zeros(8, dtype=torch.uint8, device=dev())
    off, st = i32([5]), status()
    sonic.sonic_kv4_compact(K, K, None, role, empty4(1, 1, 4, 64), empty4(1, 1, 4, 64), off,
                            k_start=i32([]), k_len=i32([]), status=st)
    assert off.tolist() == [0] and st.item() == 0
    off = i32([5, 5])
    sonic.sonic_kv4_compact(K, K, None, role, empty4(1, 1, 0, 64), empty4(1, 1, 0, 64), off,
                            k_start=i32([0]), k_len=i32([8]), status=st)
    assert off.tolist() == [0, 8] and st.item() == 4


# ------------------------------------------------------------------ decode

def check_decode(O, lse, q, K4, V4, start, lens, scale=None):
    """Against 64 bits, element by element.  With p the exact probabilities:
      O: half a bf16 step of the value (2^-8), and of sum p |V|: half an fp16 step of P (2^-11), the
         scores' error d on either side of the quotient (2 d), ex2 and the fp32 sums (2^-19);
      d: 2^-21 of the largest sum |q_d k_d| scale: the fp32 sums of a score's products, each
         addition off by at most 2^-23 of a partial sum that is no larger, and at most 4 such
         errors' worth kept in a row of 8 products' chains; q is exact to 2^-25 of its largest;
      and where P is below fp16's normal range: P = 2^(s - ref + 7) has steps of 2^-24 there, half
         a step is 2^-25 against a sum of at least 2^7 (the reference is the largest score of some
         time, so its key alone adds that much): 2^-32 of each |V|, however small p is;
      lse: d, 2^-20 of rounding in the exponents' argument, 2^-21 of lse."""
    nl, B, hq, d_ = q.shape
    K, V = plain.decode(*K4).transpose(1, 2), plain.decode(*V4).transpose(1, 2)
    scale = scale or 1 / d_ ** 0.5
    for l in range(nl):
        for b in range(B):
            rows = slice(start[b], start[b] + lens[b])
            o, z, size, big = plain.attend(q[l, b].to(F), K[l, rows], V[l, rows], scale)
            err = big * 2.0 ** -21
            tol = 2.0 ** -8 * o.abs() + (2.0 ** -11 + 2 * err + 2.0 ** -19) * size
            tol += 2.0 ** -32 * V[l, rows].abs().sum(0).repeat_interleave(hq // V.shape[2], 0)
            diff = (O[l, b].to(F) - o).abs()
            assert bool((diff <= tol).all()), (l, b, lens[b], float((diff - tol).max()))
            if lse is not None:
                if lens[b] == 0:
                    assert bool((lse[l, b] == -torch.inf).all())
                else:
                    dz = (lse[l, b].to(F) - z).abs()
                    assert bool((dz <= err + 2.0 ** -20 + 2.0 ** -21 * z.abs()).all()), (l, b, float(dz.max()))


def layout(lens, gap=5):
    start, at = [], 2
    for n in lens:
        start.append(at)
        at += n + gap
    return start, at


def cache_with_garbage(nl, hkv, rows, d, start, lens, seed):
    """Random four-bit rows; rows outside the sequences hold scale bytes that are NaN."""
    K4, V4 = random4(nl, hkv, rows, d, seed), random4(nl, hkv, rows, d, seed + 1)
    out = torch.ones(rows, dtype=torch.bool)
    for s, n in zip(start, lens):
        out[s:s + n] = False
    K4[1][:, :, out.to(dev())], V4[1][:, :, out.to(dev())] = 255, 255
    return K4, V4


HEADS = [(1, 1, 64), (2, 1, 64), (32, 8, 64), (24, 2, 64), (8, 2, 128), (7, 7, 128), (28, 4, 128), (16, 1, 128),
         (9, 1, 128)]


@pytest.mark.parametrize("hq,hkv,d", HEADS)
@pytest.mark.parametrize("lens", [[1], [0, 1, 15, 16, 17, 31, 33, 0], [127, 128, 129, 1000], [2500, 3, 640]])
def test_decode(hq, hkv, d, lens):
    nl = 2
    start, rows = layout(lens)
    K4, V4 = cache_with_garbage(nl, hkv, rows, d, start, lens, seed=hq + len(lens))
    q = inputs.randn((nl, len(lens), hq, d), 11, device=dev()) * 1.5
    O = torch.full_like(q, float("nan"))
    lse = torch.full((nl, len(lens), hq), float("nan"), device=dev())
    st = status()
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=max(lens), lse=lse, status=st)
    assert st.item() == 0
    check_decode(O, lse, q, K4, V4, start, lens)


@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (16, 2, 64)])
def test_decode_extreme_queries_and_scales(hq, hkv, d):
    """Heads whose queries are tiny, huge or zero (the power of two they are scaled by), scale
    bytes from end to end, a softmax_scale of its own."""
    lens = [200, 33]
    start, rows = layout(lens)
    K4 = random4(1, hkv, rows, d, 1, 0, 227)
    V4 = random4(1, hkv, rows, d, 2, 0, 227)
    q = inputs.randn((1, 2, hq, d), 11, device=dev())
    mult = torch.logspace(-30, -6, hq, device=dev())
    mult[0], mult[1] = 0.0, 1e-38
    q = (q.float() * mult[:, None]).to(torch.bfloat16)
    O, lse = torch.empty_like(q), torch.empty((1, 2, hq), device=dev())
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=200, lse=lse,
                                softmax_scale=0.3)
    check_decode(O, lse, q, K4, V4, start, lens, scale=0.3)


@pytest.mark.parametrize("hq,hkv,d,seqs,longest", [(8, 2, 64, 1500, 40), (4, 4, 128, 700, 150), (12, 1, 128, 1030, 90)])
def test_decode_many_short_sequences(hq, hkv, d, seqs, longest):
    """More sequences than a block keeps in shared memory, several per warp, some empty."""
    rng = np.random.default_rng(seqs)
    lens = rng.integers(0, longest + 1, seqs).tolist()
    lens[seqs // 2] = 900  # and one that is cut
    start, rows = layout(lens, gap=1)
    K4, V4 = cache_with_garbage(1, hkv, rows, d, start, lens, seed=3)
    q = inputs.randn((1, seqs, hq, d), 5, device=dev())
    O, lse = torch.empty_like(q), torch.empty((1, seqs, hq), device=dev())
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=900, lse=lse)
    check_decode(O, lse, q, K4, V4, start, lens)


def test_decode_many_layers_of_short_sequences():
    """Long shares of short sequences: a warp for each, cut ones among them."""
    nl, hq, hkv, d = 8, 8, 1, 128
    rng = np.random.default_rng(2)
    lens = rng.integers(1, 129, 800).tolist()
    start, rows = layout(lens, gap=0)
    K4, V4 = random4(nl, hkv, rows, d, 3), random4(nl, hkv, rows, d, 4)
    q = inputs.randn((nl, 800, hq, d), 5, device=dev())
    O, lse = torch.empty_like(q), torch.empty((nl, 800, hq), device=dev())
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=128, lse=lse)
    check_decode(O[:1], lse[:1], q[:1], (K4[0][:1], K4[1][:1]), (V4[0][:1], V4[1][:1]), start, lens)
    check_decode(O[-1:], lse[-1:], q[-1:], (K4[0][-1:], K4[1][-1:]), (V4[0][-1:], V4[1][-1:]), start, lens)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_decode_equal_shares(hq, hkv, d):
    """Sequences long enough that no cluster of blocks takes them: cut between blocks, several to a
    block, empty ones, and short ones that single warps take."""
    lens = [90_000, 0, 17, 4000, 1, 130, 128, 2300, 60, 0, 33]
    start, rows = layout(lens)
    K4, V4 = cache_with_garbage(2, hkv, rows, d, start, lens, seed=hq)
    q = inputs.randn((2, len(lens), hq, d), 11, device=dev())
    O = torch.full_like(q, float("nan"))
    lse = torch.full((2, len(lens), hq), float("nan"), device=dev())
    st = status()
    ws = None
    for _ in range(2):  # the second call with the first one's workspace
        ws = sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=90_000, lse=lse,
                                         status=st, workspace=ws)
    assert st.item() == 0
    check_decode(O, lse, q, K4, V4, start, lens)


@pytest.mark.parametrize("hq,hkv,d", [(28, 4, 128), (16, 1, 64)])
@pytest.mark.parametrize("batch,longest", [(1, 700), (3, 5000), (40, 300), (170, 200)])
def test_decode_clusters_of_every_size(hq, hkv, d, batch, longest):
    """One to eight blocks to a sequence and KV head, lengths that leave blocks without keys."""
    rng = np.random.default_rng(batch)
    lens = rng.integers(0, longest, batch).tolist()
    lens[0] = longest
    start, rows = layout(lens)
    K4, V4 = cache_with_garbage(1, hkv, rows, d, start, lens, seed=batch)
    q = inputs.randn((1, batch, hq, d), 3, device=dev())
    O, lse = torch.full_like(q, float("nan")), torch.empty((1, batch, hq), device=dev())
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=longest, lse=lse)
    check_decode(O, lse, q, K4, V4, start, lens)


@pytest.mark.parametrize("hq,hkv,d", HEADS)
def test_decode_a_warp_each(hq, hkv, d):
    """Units enough for all warps: lengths around the tiles, empty sequences, one that lies outside."""
    lens = [0, 1, 15, 16, 17, 47, 48, 49, 33, 0, 96, 5] * 50
    nl, cap = max(1, 4 // hkv), 90  # (the longest are cut to 90)
    kept = [min(n, cap) for n in lens]
    start, rows = layout(kept, gap=2)
    K4, V4 = cache_with_garbage(nl, hkv, rows, d, start, kept, seed=d)
    q = inputs.randn((nl, len(lens), hq, d), 9, device=dev())
    O = torch.full_like(q, float("nan"))
    lse = torch.full((nl, len(lens), hq), float("nan"), device=dev())
    st = status()
    at = list(start)
    at[3], kept[3] = rows - 5, 0  # 16 rows from there end outside the cache: refused
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(at), max_len=cap, lse=lse, status=st)
    assert st.item() != 0
    check_decode(O, lse, q, K4, V4, start, kept)


@pytest.mark.parametrize("hq,hkv,d", [(4, 4, 64), (8, 1, 128)])
def test_decode_equal_shares_of_many_sequences(hq, hkv, d):
    """More sequences than a block of equal shares keeps in shared memory."""
    rng = np.random.default_rng(hq)
    lens = rng.integers(0, 120, 1100).tolist()
    lens[400], lens[1099] = 3000, 0
    start, rows = layout(lens)
    K4, V4 = cache_with_garbage(1, hkv, rows, d, start, lens, seed=d)
    q = inputs.randn((1, len(lens), hq, d), 9, device=dev())
    O = torch.full_like(q, float("nan"))
    lse = torch.full((1, len(lens), hq), float("nan"), device=dev())
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=3000, lse=lse)
    check_decode(O, lse, q, K4, V4, start, lens)


def test_decode_refused_and_clipped_sequences():
    hq, hkv, d = 8, 2, 128
    K4, V4 = random4(1, hkv, 100, d, 1), random4(1, hkv, 100, d, 2)
    q = inputs.randn((1, 3, hq, d), 5, device=dev())
    for start, lens, max_len in (([0, 90, 20], [30, 11, 7], 64), ([0, -1, 20], [30, 4, 7], 64)):
        O, st = torch.full_like(q, 9.0), status()
        sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=max_len, status=st)
        assert st.item() == 1
        lens[1] = 0
        check_decode(O, None, q, K4, V4, [max(s, 0) for s in start], lens)
    O, st = torch.full_like(q, 9.0), status()
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32([30, 50, 7]), O, kv_start=i32([0, 30, 20]), max_len=40, status=st)
    assert st.item() == 1
    check_decode(O, None, q, K4, V4, [0, 30, 20], [30, 40, 7])


def test_decode_strides_workspace_and_empty_cache():
    nl, hq, hkv, d, lens = 3, 8, 2, 64, [70, 300]
    start, rows = layout(lens)
    wide = [random4(nl, hkv + 1, rows, d, 3 + i) for i in range(2)]  # layers further apart than packed
    K4, V4 = (tuple(x[:, :hkv] for x in w) for w in wide)
    qb = inputs.randn((nl, 3, hq, d), 5, device=dev())
    ob = torch.full_like(qb, 4.0)
    q, O = qb[:, :2], ob[:, :2]
    ws = torch.empty(1 << 22, dtype=torch.uint8, device=dev())[5:]
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=300, workspace=ws)
    check_decode(O, None, q, K4, V4, start, lens)
    assert bool((ob[:, 2] == 4).all())
    O2, lse = torch.full_like(q, 3.0).contiguous(), torch.zeros((nl, 2, hq), device=dev())
    sonic.sonic_attn_decode_kv4(q, empty4(nl, hkv, 0, d), empty4(nl, hkv, 0, d), i32([0, 0]), O2,
                                kv_start=i32([0, 0]), max_len=0, lse=lse)
    assert bool((O2 == 0).all()) and bool((lse == -torch.inf).all())


def test_decode_far_rows():
    """Byte offsets past 2^31 and 2^32 within one head's rows."""
    rows, hq, hkv, d = 70_000_000, 4, 1, 128
    K4, V4 = empty4(1, hkv, rows, d), empty4(1, hkv, rows, d)
    lens, start = [50, 300], [35_000_000, rows - 300]
    for s, n in zip(start, lens):
        for X, seed in ((K4, 1), (V4, 2)):
            c, sc = random4(1, hkv, n, d, seed + n)
            X[0][:, :, s:s + n], X[1][:, :, s:s + n] = c, sc
    q = inputs.randn((1, 2, hq, d), 5, device=dev())
    O, lse = torch.empty_like(q), torch.empty((1, 2, hq), device=dev())
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32(lens), O, kv_start=i32(start), max_len=300, lse=lse)
    near = [tuple(torch.cat([x[:, :, s:s + n] for s, n in zip(start, lens)], 2) for x in X) for X in (K4, V4)]
    check_decode(O, lse, q, near[0], near[1], [0, 50], lens)
    # and the same rows packed there and read from there
    Kn = inputs.randn((1, 3, hkv, d), 8, device=dev())
    at = i32([rows - 1, 0, 40_000_000])
    out = [torch.zeros_like(Kn) for _ in range(2)]
    sonic.sonic_kv4_store(Kn, Kn, K4, V4, dst_row=at)
    sonic.sonic_kv4_load(K4, V4, *out, src_row=at)
    want = plain.decode(*plain.encode(Kn))
    assert torch.equal(out[0].cpu().double(), want) and torch.equal(out[1].cpu().double(), want)


def test_captured_twice_on_another_stream():
    """store, load and decode in two graphs with workspaces of their own, replayed side by side,
    and an eager call on a stream that is not the current one."""
    hq, hkv, d, n = 28, 4, 128, 700
    graphs, keep = [], []
    for k in range(2):
        K, V = (inputs.randn((1, n, hkv, d), 10 * k + j, device=dev()) for j in range(2))
        K4, V4 = empty4(1, hkv, n, d), empty4(1, hkv, n, d)
        q = inputs.randn((1, 1, hq, d), 33 + k, device=dev())
        O, lens, start = torch.zeros_like(q), i32([n]), i32([0])
        oK, oV = torch.zeros_like(K), torch.zeros_like(V)
        ws = sonic.sonic_attn_decode_kv4(q, K4, V4, lens, O, kv_start=start, max_len=n)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            sonic.sonic_kv4_store(K, V, K4, V4)
            sonic.sonic_attn_decode_kv4(q, K4, V4, lens, O, kv_start=start, max_len=n, workspace=ws)
            sonic.sonic_kv4_load(K4, V4, oK, oV)
        graphs.append(g)
        keep.append((K, V, K4, V4, q, O, oK, oV, ws, lens, start))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        graphs[0].replay()
        with torch.cuda.stream(side):
            graphs[1].replay()
    torch.cuda.synchronize()
    for K, V, K4, V4, q, O, oK, oV, *_ in keep:
        assert torch.equal(oK.cpu().double(), plain.decode(*plain.encode(K)))
        check_decode(O, None, q, K4, V4, [0], [n])
    K, V, K4, V4, q, O, *_ = keep[0]
    O2 = torch.zeros_like(O)
    side.wait_stream(torch.cuda.current_stream())
    sonic.sonic_attn_decode_kv4(q, K4, V4, i32([n]), O2, kv_start=i32([0]), max_len=n, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(O, O2)


def test_binding_refuses():
    hkv, d, rows = 2, 64, 12
    K = inputs.randn((2, rows, hkv, d), 1, device=dev())
    K4, V4 = empty4(2, hkv, rows, d), empty4(2, hkv, rows, d)
    bad = [dict(K=K.half()), dict(K=K.cpu()), dict(V=K[:1]), dict(K=K.transpose(1, 2)), dict(V=K[:, :5]),
           dict(K4=(K4[0], K4[1][..., :2])), dict(K4=(K4[0][:, :1], K4[1])), dict(V4=(V4[0].char(), V4[1])),
           dict(src_row=i32([0, 1]).long()), dict(src_row=i32([0, 1]), n_rows=3),
           dict(dst_row=i32([0, 1, 2, 3])[::2]), dict(status=torch.zeros(1, device=dev()))]
    for kw in bad:
        a = dict(K=K, V=K, K4=K4, V4=V4)
        a.update({k: kw.pop(k) for k in list(kw) if k in a})
        with pytest.raises(sonic.SonicError):
            sonic.sonic_kv4_store(a["K"], a["V"], a["K4"], a["V4"], **kw)
    q = inputs.randn((2, 3, 4, d), 1, device=dev())
    ok = dict(q=q, lens=i32([1, 2, 3]), O=torch.empty_like(q), kv_start=i32([0, 2, 4]), lse=None, status=None)
    for kw in (dict(q=q[..., :32].contiguous()), dict(q=q[:1]), dict(O=q[:, :2].contiguous()),
               dict(lens=i32([1, 2])), dict(kv_start=i32([0])), dict(lse=torch.empty((2, 3, 5), device=dev())),
               dict(O=q.float())):
        a = {**ok, **kw}
        with pytest.raises(sonic.SonicError):
            sonic.sonic_attn_decode_kv4(a["q"], K4, V4, a["lens"], a["O"], kv_start=a["kv_start"], max_len=5,
                                        lse=a["lse"])


def test_what_stands_beside_an_infinity():
    """An infinity's block has the largest scale, 10240: what lies beside it keeps a code from a quarter of that on."""
    row = [float("inf"), 20000.0, 2560.0, 2576.0, -2560.0, -2576.0, 7680.0, 7712.0, 61440.0, 3e38, -3e38, 1.0, 0.0, 12800.0,
           17920.0, -float("inf")]
    K = torch.tensor(row * 4, dtype=torch.bfloat16, device=dev()).view(1, 1, 1, 64)
    K4, V4 = empty4(1, 1, 1, 64), empty4(1, 1, 1, 64)
    oK, oV = torch.empty_like(K), torch.empty_like(K)
    sonic.sonic_kv4_store(K, K, K4, V4)
    sonic.sonic_kv4_load(K4, V4, oK, oV)
    assert bool((K4[1] == 226).all())
    want = plain.decode(*plain.encode(K.transpose(1, 2))).transpose(1, 2)
    assert torch.equal(oK.cpu().double(), want) and torch.equal(oV.cpu().double(), want)
    assert want.flatten()[:6].tolist() == [61440, 20480, 0, 5120, 0, -5120]
