"""Launches of the calls around a layer's attention, and calls of their Python forms, that other tests pass over.  No device."""
import pytest

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
