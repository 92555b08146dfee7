"""Launches of the calls around a layer's attention, and calls of their Python forms, that other tests pass over.  No device."""
import pytest
import torch

import paper_2406_03488_amd as s1f
from paper_2406_03488_amd import binding
from test_host_layer import good
from test_host_layer_launches import launches, of


@pytest.mark.parametrize("shape", [(16384, 1024, 65536), (2048, 2048, 131072), (30000, 64, 20000), (65, 8192, 32768), (4099, 4096, 11008), (1, 4096, 11008)])
def test_fp32_sums_between_the_projections_are_short(tmp_path, shape):
    """y's and dx's sums have fewer than 12288 terms: a launch for each turn, its tiles in parts or not."""
    n, h, f = shape
    done = launches(tmp_path, [("ffn", n, h, f, 0)])
    for kernel, terms in (("Lb0ELb0E", f), ("Lb0ELb1E", 2 * f)):
        turns = [(name, grid) for name, grid in of(done, "ffn_product") if kernel in name]
        if not turns:
            assert n <= 16 and kernel == "Lb0ELb0E"     # (the kernel of few rows: eight waves, a part each)
            continue
        name, grid = turns[0]
        bm, bn = next((m, c) for m, c in ((256, 256), (128, 128), (64, 128)) if f"Li{m}ELi{c}" in name)
        tiles = -(-n // bm) * -(-h // bn)
        parts = grid // tiles if grid % tiles == 0 else 1     # (else whole tiles are among them)
        assert -(-terms // len(turns)) // parts < 12288 + 64, (kernel, len(turns), parts)
        # (the first turn writes, the others add)
        assert ["ResultE1" in name for name, _ in turns] == [True] + [False] * (len(turns) - 1) and all(g == grid for _, g in turns)
    assert not [1 for name, _ in of(launches(tmp_path, [("ffn", n, h, f, 1)]), "ffn_product") if "Lb0" in name and "ResultE2" in name]


@pytest.mark.parametrize("name,positions,values", [("rope_fwd", 6, (2, 10)), ("rope_bwd", 6, (2, 10)), ("qk_norm_rope_fwd", 9, (2, 13)), ("qk_norm_rope_bwd", 11, (2, 15))])
def test_a_first_position_reaches_the_library(monkeypatch, name, positions, values):
    """An integer in the place of the positions' tensor, with values and without."""
    calls = []

    class Library:
        def __getattr__(self, entry):
            return lambda *args: calls.append((entry, args)) or 0
    monkeypatch.setattr(binding, "load_library", Library)
    monkeypatch.setattr(binding, "_stream_ptr", lambda: 0)
    monkeypatch.setattr(binding, "_check_device", lambda *t: None)
    monkeypatch.setattr(binding, "_native", lambda: binding._PythonForms)
    args = good()[name]
    assert isinstance(args[positions], torch.Tensor) and args[positions + 1] == 3
    tensor = args[positions].data_ptr()
    getattr(s1f, name)(*args)
    args[positions] = -77
    getattr(s1f, name)(*args)
    for i in values:
        args[i] = None
    getattr(s1f, name)(*args)
    assert [entry for entry, _ in calls] == ["s1f_" + name] * 3
    # (positions, their stride, the first row's, seg_off) behind the magnitude
    for (_, got), want in zip(calls, ((tensor, 5, 0, 3), (None, 0, -77, 3), (None, 0, -77, 3))):
        at = next(i for i in range(len(got)) if got[i:i + 4] == want)
        assert got[at - 1] == 1.0


def test_a_tensor_in_the_place_of_the_segments_first_row_is_refused(monkeypatch):
    monkeypatch.setattr(binding, "_check_device", lambda *t: None)
    monkeypatch.setattr(binding, "_native", lambda: binding._PythonForms)
    for name, positions in (("rope_fwd", 6), ("rope_bwd", 6), ("qk_norm_rope_fwd", 9), ("qk_norm_rope_bwd", 11)):
        args = good()[name]
        args[positions + 1] = args[positions]
        with pytest.raises((TypeError, ValueError)):
            getattr(s1f, name)(*args)


def test_turns_of_y_and_dx_take_tiles_of_every_size(tmp_path):
    """tests/test_gpu_ffn_spread.py checks the values of these."""
    from test_gpu_ffn_spread import TURNS
    kinds = set()
    for shape in TURNS:
        done = launches(tmp_path, [("ffn", *shape, 0)])
        for (name, *_), (behind, *_) in zip(done, done[1:] + [("", 0, 0, 0)]):
            if "ffn_product" in name and "ResultE2" in name and "Lb1ELb1E" not in name:
                side = next(s for s in ("256ELi256", "128ELi128", "64ELi128") if f"Li{s}" in name)
                kinds.add(("y" if "Lb0ELb0E" in name else "dx", side, "join" in behind))
    assert {(k, s, True) for k in ("y", "dx") for s in ("256ELi256", "128ELi128", "64ELi128")} <= kinds and {("y", "256ELi256", False), ("dx", "256ELi256", False)} <= kinds, kinds
