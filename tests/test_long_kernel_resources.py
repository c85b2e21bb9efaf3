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
