"""Registers and spills of the serving kernels for shared and long contexts and
of the products in 8-bit integers."""
import re

from test_kernel_resources import kernels  # noqa: F401  (a fixture)


def test_registers(kernels):  # noqa: F811
    """The workgroups that a compute unit is to hold (256 threads: 512 registers a
    lane for one, 256 for two, 168 for three), without spills: of the attention by
    waves up to 16 rows, the selection, the products and the joins."""
    most = {"k_linear_fewILi.ELi.ELi.E": 128, "k_linear_tilesILi.ELi4ELi4ELb0E": 512, "k_linear_tilesILi.ELi2ELi2E": 256, "k_linear_joinILi": 128,
            "k_quantizeILi": 128, "k_sharedILi.ELi64ELi1ELi1E": 256, "k_sharedILi.ELi128ELi1ELi1E": 256, "k_sharedILi.ELi256ELi1ELi1E": 512,
            "k_shared_joinILi": 128, "k_boundsILi": 128, "k_scoresILi": 128, "k_scores_manyILi.ELi(64|128)E": 256,
            "k_scores_manyILi.ELi256E": 512, "k_pickILi": 128, "k_selected_joinILi": 128, "k_selectedILi.ELi64E": 168,
            "k_selectedILi.ELi256E": 512}
    for pattern, vgprs in most.items():
        found = {k: v for k, v in kernels.items() if re.search(pattern, k)}
        assert found, pattern
        for name, (used, spills) in found.items():
            assert used <= vgprs and spills == 0, (name, used, spills)
    # Three workgroups a unit at heads of 128 cost a few spilled registers.
    for name, (used, spills) in kernels.items():
        if re.search("k_selectedILi.ELi128E", name):
            assert used <= 168 and spills <= 8, (name, used, spills)


def test_shared_passes_registers(kernels):  # noqa: F811
    """Every pair of passes of the attention over a shared prefix. Both are in one
    kernel, at two workgroups a compute unit (one at heads of 256): with passes of 128
    rows, and two of 32, registers are spilled, no more than here."""
    spilled = {   # head_dim: {(prefix's rows, own rows): registers}
        64: {}, 128: {(2, 2): 48, (8, 1): 72, (8, 2): 112, (8, 8): 184}, 256: {(2, 2): 48, (8, 1): 136, (8, 2): 176, (8, 8): 304}}
    for D, known in spilled.items():
        for pair in ((1, 1), (2, 1), (8, 1), (2, 2), (8, 2), (8, 8)):
            found = {k: v for k, v in kernels.items() if re.search(f"k_sharedILi.ELi{D}ELi{pair[0]}ELi{pair[1]}E", k)}
            assert len(found) == 2   # both types
            for name, (used, spills) in found.items():
                assert used <= (512 if D == 256 else 256) and spills <= known.get(pair, 0), (name, used, spills)
