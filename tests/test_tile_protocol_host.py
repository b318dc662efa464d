"""The order of events around one row group of the attention tiles, as a model run under random schedules.

Two softmax warps hold the two halves of a row's keys; a third actor makes scores and products.  The model has the
rules that the kernel keeps: whose words are written when, what waits for what, and how a warp leaves.  Under them
no schedule may read a word that is not its tile's, or leave a warp waiting; without any one of them some schedule does."""
import os
import random

import pytest


def run(seed, tiles, buffers, words, farewell, give_up=None, together=True):
    """Errors of one random schedule.  buffers: score buffers of the row tile (scores run that many tiles ahead); words:
    sets of words that maxima are exchanged through; farewell: a leaving warp meets its partner and says so, else it
    only arrives once where a wait gave up; give_up = (half, tile): the wait that gives up; together: the halves
    meet again after rescaling their columns of the result, which the products of either half's weights add to."""
    rng = random.Random(seed)
    scores, weights, products = set(), set(), set()
    top, errors, dead = {}, set(), [False]
    meeting = dict(sides=[], turn=0, gone={})
    rescaling = [False, False]

    def side(leaving):
        turn = meeting["turn"]
        meeting["sides"].append(leaving)
        if len(meeting["sides"]) == 2:
            meeting["gone"][turn] = any(meeting["sides"])
            meeting["sides"], meeting["turn"] = [], turn + 1
        return turn

    def meet(leaving=False):
        turn = side(leaving)
        while meeting["turn"] == turn:
            yield "wait"
        return farewell and meeting["gone"][turn]

    def softmax(half):
        parted, ok = False, True
        for i in range(tiles):
            if give_up == (half, i):
                dead[0] = True
            while i not in scores and not dead[0]:
                yield "wait"
            if i not in scores or give_up == (half, i):
                ok = False
                break
            yield
            top[i % words, half] = i
            yield
            parted = yield from meet()
            if parted:
                ok = False
                break
            yield
            if top.get((i % words, half ^ 1)) != i and not dead[0]:
                errors.add("maximum of another tile")
            if i % 3:   # the maximum has moved
                while buffers == 2 and i - 1 not in products and not dead[0]:
                    yield "wait"
                if buffers == 2 and i - 1 not in products:
                    ok = False
                    break
                rescaling[half] = True
                for _ in range(rng.randint(1, 6)):
                    yield
                rescaling[half] = False
                if together:
                    parted = yield from meet()
                    if parted:
                        ok = False
                        break
            for _ in range(rng.randint(1, 4)):
                yield
            weights.add((i, half))
        if ok:
            parted = yield from meet()   # the sums of the segment
        if farewell:
            if not parted:
                yield from meet(True)
        elif dead[0]:
            side(True)

    def matrix():
        for i in range(min(buffers, tiles)):
            yield
            scores.add(i)
        for i in range(tiles):
            for half in (0, 1):
                while (i, half) not in weights:
                    if dead[0]:
                        return
                    yield "wait"
                for _ in range(2):
                    yield
                    if any(rescaling):
                        errors.add("products while columns are rescaled")
            products.add(i)
            if i + buffers < tiles:
                yield
                scores.add(i + buffers)

    actors = [softmax(0), softmax(1), matrix()]
    rng.shuffle(actors)
    idle = 0
    while actors and idle < 300:
        k = rng.randrange(len(actors)) if rng.random() < 0.5 else 0   # one actor is favoured
        try:
            idle = idle + 1 if next(actors[k]) == "wait" else 0
        except StopIteration:
            del actors[k]
            idle = 0
    if actors:
        errors.add("a warp waits for ever")
    return errors


def over_schedules(n, **kw):
    found = set()
    for seed in range(n):
        found |= run(seed, 6, **kw)
    return found


@pytest.mark.parametrize("buffers", [1, 2])
def test_no_schedule_goes_wrong(buffers):
    assert over_schedules(1500, buffers=buffers, words=2, farewell=True) == set()
    for half in (0, 1):
        for at in range(6):
            assert over_schedules(150, buffers=buffers, words=2, farewell=True, give_up=(half, at)) == set()


def test_one_set_of_words_does_for_one_score_buffer_only():
    assert over_schedules(1500, buffers=1, words=1, farewell=True) == set()
    assert over_schedules(1500, buffers=2, words=1, farewell=True) == {"maximum of another tile"}


def test_a_single_arrival_does_not_release_the_partner_of_a_warp_that_gives_up():
    found = set()
    for half in (0, 1):
        for at in range(6):
            found |= over_schedules(150, buffers=2, words=2, farewell=False, give_up=(half, at))
    assert found == {"a warp waits for ever"}


@pytest.mark.parametrize("buffers", [1, 2])
def test_products_meet_columns_that_are_being_rescaled_unless_the_halves_meet_again(buffers):
    assert over_schedules(300, buffers=buffers, words=2, farewell=True, together=False) == {"products while columns are rescaled"}


def follow(seed, kinds, own):
    """Segments of one row tile (1) or two (2) in turn; whether the second row tile's warp gets through them.  It waits for
    phases of its scores' barrier by their parity.  own: that barrier has no phases but its own; else the odd key
    tiles of a single row tile use it too, which nobody waits for it to see, and it follows them one by one."""
    rng = random.Random(seed)
    done, ready, answered = [0], [0], [0]   # phases of the barrier; segments that the second row tile has come to; phases it saw

    def matrix():
        for i, kind in enumerate(kinds):
            while kind == 2 and ready[0] <= i:
                yield "wait"
            for tile in range(5):
                yield
                if kind == 2 or (tile % 2 and not own):
                    done[0] += 1
                    seen = done[0]
                    while kind == 2 and answered[0] < seen:
                        yield "wait"

    def second():
        parity = 0
        for i, kind in enumerate(kinds):
            ready[0] = i + 1
            for _ in range(rng.randint(0, 12)):   # writes its last result, or is held up
                yield
            for tile in range(5):
                if kind == 2 or (tile % 2 and not own):
                    while done[0] % 2 == parity:   # the phase of this parity is not over
                        yield "wait"
                    parity ^= 1
                    answered[0] = max(answered[0], done[0])

    actors, idle = [matrix(), second()], 0
    while actors and idle < 200:
        k = rng.randrange(len(actors))
        try:
            idle = idle + 1 if next(actors[k]) == "wait" else 0
        except StopIteration:
            del actors[k]
            idle = 0
    return not actors


def test_a_warp_that_nobody_waits_for_cannot_follow_phases_by_their_parity():
    kinds = [2, 1, 2, 1, 1, 2]
    assert all(follow(seed, kinds, own=True) for seed in range(2000))
    assert not all(follow(seed, kinds, own=False) for seed in range(2000))


def test_tensor_memory_is_not_held_while_waiting_for_the_kernel_before():
    """Where two kernels overlap on an SM, one that waits for the other to end must not hold what the other may still
    ask for."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "paper_2609_11744_b200", "csrc", "kvc_attention_tiles.cu")) as f:
        kernel = f.read().split("kvc_attn_tiles_kernel(const __grid_constant__", 1)[1]
    assert 0 < kernel.index("kvc_pdl_begin(") < kernel.index("tcgen05.alloc")
