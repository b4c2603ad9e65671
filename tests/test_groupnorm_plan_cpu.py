"""The group norm's blocks of channels (gn_plan in csrc/groupnorm.hip) for every width and number of groups, on the CPU."""
import numpy as np
import pytest

MOST = 16384  # channels
THREADS = 256


def blocks(G, Cg, kg, VE):
    """gn_blocks for arrays G, Cg and kg: groups per block."""
    kg = -(-G // -(-G // kg))
    while True:
        more = (kg < G) & ((G - (-(-G // kg) - 1) * kg) * Cg < VE)
        if not more.any():
            return kg
        kg = kg + more


@pytest.mark.parametrize("VE", [4, 8])
def test_blocks_fit_a_wave_and_hold_a_vector(VE):
    CB = 64 * VE
    for Cg in range(1, CB + 1):
        G = np.arange(1, MOST // Cg + 1)
        G = G[G * Cg >= VE]  # (narrower rows are one block, element by element)
        kg = blocks(G, Cg, np.full_like(G, min(CB // Cg, THREADS)), VE)
        last = G - (-(-G // kg) - 1) * kg
        assert (kg * Cg <= CB).all() and (kg <= THREADS).all()
        assert ((last > 0) & (last <= kg) & (last * Cg >= VE)).all()


@pytest.mark.parametrize("VE", [4, 8])
def test_pieces_of_wide_groups_hold_a_vector(VE):
    CB = 64 * VE
    Cg = np.arange(CB + 1, MOST + 1)
    pieces = -(-Cg // CB)
    width = -(-Cg // pieces)
    assert (width <= CB).all() and (Cg - (pieces - 1) * width >= VE).all()
