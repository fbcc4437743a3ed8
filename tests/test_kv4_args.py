"""Four-bit caches, key mass and eviction without a GPU: struct layouts, what the host refuses
before anything is launched, and the plain forms the GPU tests compare with."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2601_21927_gb300 import sonic
from tests import kv4_plain as plain

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
by = ctypes.byref


def test_struct_layout_matches_c(tmp_path):
    names = ["sonic_kv4_cache", "sonic_kv4_rows_args", "sonic_kv4_compact_args", "sonic_decode_kv4_args",
             "sonic_key_mass_args", "sonic_evict_part", "sonic_evict_args"]
    src = ['#include <stdio.h>', '#include <stddef.h>', '#include "sonic.h"', 'int main(void){']
    for name in names:
        src.append(f'printf("{name} %zu\\n", sizeof({name}));')
        for f, _ in getattr(sonic, name)._fields_:
            src.append(f'printf("{name}.{f} %zu\\n", offsetof({name}, {f}));')
    src.append("return 0;}")
    c = tmp_path / "layout.c"
    c.write_text("\n".join(src))
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(ROOT, "include"), str(c), "-o", str(exe)], check=True)
    out = dict(x.split() for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                                 check=True).stdout.splitlines())
    for name in names:
        cls = getattr(sonic, name)
        assert int(out[name]) == ctypes.sizeof(cls), name
        for f, _ in cls._fields_:
            assert int(out[f"{name}.{f}"]) == getattr(cls, f).offset, f"{name}.{f}"


def cache(**kw):
    c = sonic.sonic_kv4_cache(16, 16, 16, 16, 8, 4096, 512)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CACHES = [dict(k_codes=None), dict(k_scales=None), dict(k_codes=24), dict(k_scales=20), dict(rows=-1)]


def test_rows_refusals():
    lib = sonic.load()
    for call in (lambda c, a, k=16, v=16: lib.sonic_kv4_store(k, v, c and by(c), a and by(a), None),
                 lambda c, a, k=16, v=16: lib.sonic_kv4_load(c and by(c), k, v, a and by(a), None)):
        def args(**kw):
            a = sonic.sonic_kv4_rows_args(2, 2, 128, 4, None, None, None, 8, 2048, None)
            for k, v in kw.items():
                setattr(a, k, v)
            return a
        assert call(None, args()) == 1 and call(cache(), None) == 1
        assert call(cache(), args(n_rows=0)) == 0  # nothing to do
        for kw in (dict(n_layers=0), dict(n_heads_kv=0), dict(n_rows=-1), dict(total_rows=-1),
                   dict(kv_layer_stride=0), dict(kv_layer_stride=2044)):
            assert call(cache(), args(**kw)) == 1, kw
        for d in (0, 32, 96, 256):
            assert call(cache(), args(head_dim=d)) == 2
        assert call(cache(), args(), None) == 1 and call(cache(), args(), 16, None) == 1
        assert call(cache(), args(), 24) == 1 and call(cache(), args(), 16, 8) == 1
        for kw in BAD_CACHES + [dict(v_codes=None), dict(v_scales=8), dict(codes_layer_bytes=0),
                                dict(codes_layer_bytes=24), dict(scales_layer_bytes=4)]:
            assert call(cache(**kw), args()) == 1, kw


def test_compact_refusals():
    lib = sonic.load()

    def call(c=None, K=16, V=16, role=16, offsets=16, **kw):
        a = sonic.sonic_kv4_compact_args(2, 2, 2, 128, 16, 16, None, 8, 2048)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.sonic_kv4_compact(K, V, None, role, by(c or cache()), offsets, by(a), None)

    assert lib.sonic_kv4_compact(16, 16, None, 16, by(cache()), 16, None, None) == 1
    for kw in (dict(batch=-1), dict(n_layers=0), dict(n_heads_kv=0), dict(k_start=None), dict(k_len=None),
               dict(total_rows=0), dict(kv_layer_stride=4), dict(K=None), dict(V=None), dict(K=8),
               dict(role=None), dict(offsets=None)):
        assert call(**kw) == 1, kw
    for kw in BAD_CACHES:
        assert call(cache(**kw)) == 1, kw
    assert call(head_dim=96) == 2 and call(batch=65536) == 2
    assert call() == 3  # no workspace


def test_decode_refusals():
    lib = sonic.load()

    def call(c=None, q=16, lens=16, O=16, **kw):
        a = sonic.sonic_decode_kv4_args(2, 2, 8, 2, 128, 16, 64, 2048, 2048)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.sonic_attn_decode_kv4(q, by(c or cache()), lens, O, by(a), None)

    assert lib.sonic_attn_decode_kv4(16, by(cache()), 16, 16, None, None) == 1
    for kw in (dict(batch=-1), dict(n_layers=0), dict(n_heads_q=7), dict(n_heads_kv=0), dict(max_len=-1),
               dict(kv_start=None), dict(q=None), dict(lens=None), dict(O=None), dict(q=8), dict(O=18),
               dict(q_layer_stride=12), dict(o_layer_stride=3)):
        assert call(**kw) == 1, kw
    for kw in BAD_CACHES + [dict(v_codes=None)]:
        assert call(cache(**kw)) == 1, kw
    assert call(head_dim=80) == 2 and call(n_heads_q=34) == 2  # 17 heads a group
    assert call() == 3 and call(batch=0) == 0


def test_key_mass_refusals():
    lib = sonic.load()

    def call(q=16, K=16, c=None, lse=16, lens=16, mass=16, **kw):
        a = sonic.sonic_key_mass_args(2, 2, 8, 2, 128, 16, 64, 8, 2048, 16, 16, 4, 8, 8192, 0.0, 2, 2,
                                      None, 0.0, None)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.sonic_key_mass(q, K, None if c is None else by(c), lse, lens, mass, by(a), None)

    assert lib.sonic_key_mass(16, 16, None, 16, 16, 16, None, None) == 1
    for kw in (dict(batch=-1), dict(n_layers=0), dict(n_heads_q=7), dict(mass_layers=3), dict(mass_heads=0),
               dict(max_len=-1), dict(max_q_len=-1), dict(total_q_rows=-1), dict(kv_start=None),
               dict(q_start=None), dict(q_len=None), dict(q=None), dict(q=8), dict(lse=None), dict(lens=None),
               dict(mass=None), dict(K=None), dict(K=8), dict(c=cache()), dict(kv_layer_stride=12),
               dict(q_layer_stride=12), dict(K=None, c=cache(rows=9)), dict(K=None, c=cache(k_codes=24))):
        assert call(**kw) == 1, kw
    assert call(head_dim=256) == 2
    assert call(batch=0) == 0 and call(total_kv_rows=0) == 0


def test_evict_refusals():
    lib = sonic.load()

    def call(mass=16, lens=16, offsets=16, part=None, **kw):
        a = sonic.sonic_evict_args(2, 2, 2, 2, 2, 16, 64, 8, 16)
        a.out_rows, a.n_parts = 8, 1
        a.parts[0] = sonic.sonic_evict_part(16, 16, 256, 4096, 256, 512, 4096, 256, 512)
        for k, v in (part or {}).items():
            setattr(a.parts[0], k, v)
        for k, v in kw.items():
            setattr(a, k, v)
        return lib.sonic_evict_kv(mass, lens, offsets, by(a), None)

    assert lib.sonic_evict_kv(16, 16, 16, None, None) == 1
    for kw in (dict(batch=-1), dict(n_layers=0), dict(mass_layers=3), dict(mass_heads=3), dict(max_len=-1),
               dict(recent=-1), dict(out_rows=-1), dict(n_parts=5), dict(n_parts=-1), dict(mass=None),
               dict(lens=None), dict(offsets=None), dict(kv_start=None), dict(budget=None),
               dict(keep_roles=1), dict(out_role=16), dict(part=dict(src=None)), dict(part=dict(dst=None)),
               dict(part=dict(bytes=0)), dict(part=dict(bytes=6)), dict(part=dict(src=18)),
               dict(part=dict(dst_row=514)), dict(part=dict(src_head=255))):
        assert call(**kw) == 1, kw
    assert call(batch=65536) == 2
    assert call(total_kv_rows=0x7fffffff) == 2
    assert call() == 3
    assert call(workspace=24, workspace_bytes=1 << 20) == 1


def test_workspace_sizes():
    lib = sonic.load()
    assert lib.sonic_decode_kv4_workspace_size(None) == 0
    assert lib.sonic_evict_workspace_size(None) == 0
    assert lib.sonic_kv4_compact_workspace_size(None, None) == 0
    a = sonic.sonic_decode_kv4_args(0, 1, 8, 2, 128)
    assert lib.sonic_decode_kv4_workspace_size(by(a)) == 0
    a.batch, a.max_len = 4, 100
    assert lib.sonic_decode_kv4_workspace_size(by(a)) > 0


def test_binding_refuses_tensors_off_the_gpu():
    K = torch.zeros((1, 8, 2, 64), dtype=torch.bfloat16)
    four = (torch.zeros((1, 2, 8, 32), dtype=torch.uint8), torch.zeros((1, 2, 8, 4), dtype=torch.uint8))
    if torch.cuda.is_available():
        with pytest.raises(sonic.SonicError):
            sonic.sonic_kv4_store(K, K, four, four)
    else:  # no current device at all
        with pytest.raises((sonic.SonicError, RuntimeError, AssertionError)):
            sonic.sonic_kv4_store(K, K, four, four)


def test_plain_format():
    """Every border between two codes, and scale bytes from end to end, read back as they should."""
    tab = plain.scale_table()
    assert tab[226] == 10240 and tab[8] == 2.0 ** -14 and bool((tab[1:] > tab[:-1]).all())
    half = (torch.arange(227, dtype=torch.int16) << 7).view(torch.half).double()
    assert torch.equal(half, tab)
    x = torch.zeros(1, 16, dtype=torch.bfloat16)
    x[0, :8] = torch.tensor([6, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    codes, scales = plain.encode(x)
    assert scales.item() == 15 * 8  # scale 1
    got = plain.decode(codes, scales)[0, :8].tolist()
    assert got == [6, 0, 1, 1, 2, 2, 4, 4]  # ties to the even code
    # amax / 6 on a border of the scale grid: 1.0625 lies between 1 and 1.125
    y = torch.full((1, 16), 6.375, dtype=torch.bfloat16)
    assert plain.encode(y)[1].item() == 15 * 8


def test_plain_evict():
    nan = float("nan")
    assert plain.evict_rows([3, 1, 2, 2, 2], [False] * 5, 3) == [0, 2, 3]
    assert plain.evict_rows([0, nan, 0, -1.0], [False, False, True, False], 2) == [0, 2]
    assert plain.evict_rows([nan, float("-inf"), 0], [False] * 3, 2) == [0, 2]
    assert plain.evict_rows([1, 2, 3], [True, True, False], 1) == [0, 1]
    assert plain.evict_rows([], [], 4) == []


def test_evict_refuses_outputs_over_inputs():
    """Blocks write offsets, lengths and choices while others still read the lengths, starts, budgets and
    masses: an output in an input's place (whole, or by one word) is refused."""
    lib = sonic.load()
    # (name, bytes): 5 sequences, 2 x 2 choices, 40 rows in and 24 out
    ins = dict(lens=20, kv_start=20, budget=20, reserve=20, mass=640, role=40)
    outs = dict(offsets=24, out_len=20, src_idx=384, out_mass=384, out_role=96)
    place = {n: 4096 * (i + 1) for i, n in enumerate((*ins, *outs))}

    def call(**at):
        at = {**place, **at}
        a = sonic.sonic_evict_args(5, 2, 2, 2, 2, at["kv_start"], 20, 40, at["budget"], at["reserve"], at["role"], 1, 0,
                                   24, at["out_len"], at["src_idx"], at["out_mass"], at["out_role"])
        a.workspace, a.workspace_bytes, a.n_parts = 1 << 20, 1 << 16, 1
        a.parts[0] = sonic.sonic_evict_part(at.get("src", 1 << 22), 1 << 23, 256, 20480, 256, 512, 12288, 256, 512)
        return lib.sonic_evict_kv(at["mass"], at["lens"], at["offsets"], by(a), None)

    for i, n_in in ins.items():
        for o, n_out in outs.items():
            for at in (place[i], place[i] + (n_in - 4 if o != "out_role" else n_in - 1), place[i] - n_out + 4):
                assert call(**{o: at}) == 1, (i, o)
    assert call(src=1 << 23) == 1


def test_compact_refuses_outputs_over_inputs():
    lib = sonic.load()
    # 5 sequences, 40 rows in and 8 in the cache
    ins = dict(k_start=20, k_len=20, reserve=20, role=40, seg=160)
    outs = dict(offsets=24, ret_len=20, src_idx=32, out_role=8, out_seg=32)
    place = {n: 4096 * (i + 1) for i, n in enumerate((*ins, *outs))}

    def call(**at):
        at = {**place, **at}
        a = sonic.sonic_kv4_compact_args(5, 2, 2, 128, at["k_start"], at["k_len"], at["reserve"], 40, 10240,
                                         at["ret_len"], at["src_idx"], at["out_role"], at["out_seg"])
        a.workspace, a.workspace_bytes = 1 << 20, 1 << 20
        return lib.sonic_kv4_compact(1 << 22, 1 << 23, at["seg"], at["role"], by(cache()), at["offsets"], by(a), None)

    for i, n_in in ins.items():
        for o, n_out in outs.items():
            for at in (place[i], place[i] + (n_in - 4 if o != "out_role" else n_in - 1), place[i] - n_out + 4):
                assert call(**{o: at}) == 1, (i, o)


def test_key_mass_refuses_rows_beyond_32_bits():
    """A tile of 128 keys reaches past a sequence's last row: its rows still have to be 32-bit numbers."""
    lib = sonic.load()
    for rows in (2 ** 31 - 256, 2 ** 31 - 128, 2 ** 31 - 1):
        a = sonic.sonic_key_mass_args(2, 1, 8, 1, 64, 16, 64, rows, 0, 16, 16, 40, 80, 0, 0.0, 1, 1, None, 0.0, None)
        assert lib.sonic_key_mass(16, 16, None, 16, 16, 16, by(a), None) == 2
        c = sonic.sonic_kv4_cache(16, 16, None, None, rows, 0, 0)
        assert lib.sonic_key_mass(16, None, by(c), 16, 16, 16, by(a), None) == 2
