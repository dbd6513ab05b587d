"""Two warps of the linear layers' epilogue tell one another their maxima, tile by tile, through places and barriers in shared memory.
A model of that exchange is run through every order of the two warps' steps: no wait may miss its phase, and each warp must
read what the other wrote for the same tile."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2508_18182_b200", "csrc")
TILES = 6


def orders(barriers, places):
    """Every reachable state of two warps; the number of states at which a warp had a wrong value or nobody could go on."""
    # a warp: tile, step (write, tell, wait, read); a barrier: phases completed; a place: the tile whose value it holds
    start = ((0, 0), (0, 0), (0,) * barriers, (0,) * barriers, (-1,) * places, (-1,) * places)
    seen, todo, wrong = {start}, [start], 0
    while todo:
        state = todo.pop()
        moves = 0
        for me in (0, 1):
            warps, bars, held = [state[0], state[1]], [list(state[2]), list(state[3])], [list(state[4]), list(state[5])]
            tile, step = warps[me]
            if tile == TILES:
                continue
            if step == 0:
                held[me][tile % places] = tile
            elif step == 1:
                bars[1 - me][tile % barriers] += 1                    # the other's barrier, of one arrival a phase
            elif step == 2:
                # a wait for parity P goes on while the phase that runs has the other parity
                if bars[me][tile % barriers] % 2 == (tile // barriers) % 2:
                    continue
            elif held[1 - me][tile % places] != tile:
                wrong += 1
            warps[me] = (tile, step + 1) if step < 3 else (tile + 1, 0)
            moves += 1
            after = (warps[0], warps[1], tuple(bars[0]), tuple(bars[1]), tuple(held[0]), tuple(held[1]))
            if after not in seen:
                seen.add(after)
                todo.append(after)
        if moves == 0 and (state[0][0] < TILES or state[1][0] < TILES):
            wrong += 1
    return wrong


def test_two_places_and_two_barriers_are_enough():
    assert orders(2, 2) == 0
    assert orders(1, 2) > 0                                           # a warp that is a tile ahead ends a phase too early
    assert orders(2, 1) > 0


def test_the_kernel_has_two_of_each():
    text = open(os.path.join(CSRC, "dense_gemm.cu")).read()
    assert re.search(r"turn = swaps & 1u, place = turn \* 256u", text)
    assert "mbar_arrive(swap_bar(w ^ 4u, turn))" in text and "swap_bar(w, turn), (swaps >> 1) & 1u" in text
