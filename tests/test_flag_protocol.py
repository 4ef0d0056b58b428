"""The hand-over of a partial result between two blocks of the paged decode, as a model whose every interleaving is tried.

A publisher writes its partial and puts the call's number into a flag; a reader polls the flag and may give up at any
time.  A captured graph repeats the call with the same number, so after every launch the flag must hold nothing that a
later launch could take for its own: whatever the timing, a reader that accepts gets its own launch's partial."""
import pytest

CALL, GIVEN_UP, OTHER = "call", "given up", "another call's"


def _publisher(launch, clears_first=False, marks=True):
    """A generator of atomic steps on the shared memory {flag, data}."""
    def steps(m):
        if clears_first:
            m["flag"] = 0
            yield
        m["data"] = launch
        yield
        was, m["flag"] = m["flag"], CALL
        yield
        if marks and was == GIVEN_UP:
            m["flag"] = 0
    return steps


def _reader(polls, marks=True):
    """Gives up after `polls` looks."""
    def steps(m):
        for _ in range(polls):
            seen = m["flag"]
            yield
            if seen == CALL:
                break
        else:
            if marks:
                was, m["flag"] = m["flag"], GIVEN_UP
                yield
                if was != CALL:
                    m["result"] = "late"
                    return
            else:
                m["result"] = "late"
                m["flag"] = 0
                return
        m["result"] = m["data"]
        yield
        m["flag"] = 0
    return steps


def _run(order, actors, memory):
    """One interleaving: order[i] says who goes next while both can; returns the number of choices taken."""
    running = [a(memory) for a in actors]
    taken = 0
    while running:
        i = 0
        if len(running) > 1:
            i = order[taken] if taken < len(order) else 0
            taken += 1
        try:
            next(running[i])
        except StopIteration:
            running.pop(i)
    return taken


def _launches(flag, launch, make):
    """All outcomes of one launch that finds `flag`: {(result, flag behind it, data)}."""
    ends = set()
    for polls in (1, 2, 3):
        todo = [()]
        while todo:
            order = todo.pop()
            m = {"flag": flag, "data": launch - 1, "result": None}
            taken = _run(order, make(launch, polls), m)
            ends.add((m["result"], m["flag"]))
            if taken > len(order):
                todo += [order + (0,) * (k - len(order)) + (1,) for k in range(len(order), taken)]
    return ends


def _wrong(make):
    """(flag found, result, flag left) of launches that accept another launch's partial or leave something behind
    that a replay would find; follows what is left into the next launch."""
    wrong, seen, todo = set(), set(), [0, OTHER]
    while todo:
        flag = todo.pop()
        if flag in seen:
            continue
        seen.add(flag)
        for result, left in _launches(flag, 2, make):
            if result not in ("late", 2):
                wrong.add((flag, result, left))
            todo.append(left)
    return wrong, seen


def test_every_interleaving_gives_the_launchs_own_partial_or_none():
    wrong, found = _wrong(lambda launch, polls: [_publisher(launch), _reader(polls)])
    assert not wrong
    assert found == {0, OTHER}       # nothing but a cleared flag is ever left


@pytest.mark.parametrize("clears_first", [True, False])
def test_without_the_mark_of_giving_up_a_replay_takes_an_old_partial(clears_first):
    wrong, found = _wrong(lambda launch, polls: [_publisher(launch, clears_first, marks=False), _reader(polls, marks=False)])
    assert CALL in found and any(result == 1 for _, result, _ in wrong)


def test_both_outcomes_occur():
    results = {r for r, _ in _launches(0, 2, lambda launch, polls: [_publisher(launch), _reader(polls)])}
    assert results == {2, "late"}
