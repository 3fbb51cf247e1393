"""Host bookkeeping of the paged cache (no GPU): a random run of all operations against a model
that keeps every sequence's tokens and every page's contents."""
import random

import pytest

from paper_2607_27269_amd.paged import OutOfPages, PageAllocator


@pytest.mark.parametrize("seed,ps,n_pages", [(0, 1, 12), (1, 4, 20), (2, 7, 9), (3, 16, 40), (4, 3, 60)])
def test_random_run_keeps_every_token(seed, ps, n_pages):
    rng = random.Random(seed)
    a = PageAllocator(n_pages, ps)
    tokens, content = {}, {}              # sequence -> tokens; (page, row) -> token
    stamp = 0

    def copy(pairs):
        dst = [t for _, t in pairs]
        assert len(set(dst)) == len(dst) and not set(dst) & {s for s, _ in pairs}
        for s, t in pairs:
            for r in range(ps):
                content[t, r] = content.get((s, r))

    for _ in range(600):
        live = list(tokens)
        op = rng.choice(["add", "extend", "extend", "extend", "fork", "truncate", "free", "compact"])
        if op == "add" or not live:
            tokens[a.add()] = []
        elif op == "fork":
            s = rng.choice(live)
            tokens[a.fork(s)] = list(tokens[s])
        elif op == "truncate":
            s = rng.choice(live)
            n = rng.randint(0, len(tokens[s]))
            a.truncate(s, n)
            del tokens[s][n:]
        elif op == "free":
            s = rng.choice(live)
            a.free(s)
            del tokens[s]
        elif op == "compact":
            copy(a.compact())
            used = int((a.holders > 0).sum())
            assert (a.holders[:used] > 0).all()
        else:
            seqs = rng.sample(live, rng.randint(1, min(4, len(live))))
            counts = [rng.randint(0, 2 * ps) for _ in seqs]
            before = ({s: list(p) for s, p in a.pages.items()}, a.holders.copy(), sorted(a.free_pages))
            try:
                copy(a.extend(seqs, counts))
            except OutOfPages:
                assert before[0] == a.pages and (before[1] == a.holders).all() and before[2] == sorted(a.free_pages)
                continue
            for s, c in zip(seqs, counts):
                for _ in range(c):
                    n = len(tokens[s])
                    page = a.pages[s][n // ps]
                    assert a.holders[page] == 1           # a page that is written is not shared
                    stamp += 1
                    content[page, n % ps] = stamp
                    tokens[s].append(stamp)
                a.length[s] += c
        # invariants: every token is where its sequence says, every page is held or free
        held = [0] * n_pages
        for s, t in tokens.items():
            assert a.length[s] == len(t) and len(a.pages[s]) == -(-len(t) // ps)
            assert [content[a.pages[s][i // ps], i % ps] for i in range(len(t))] == t
            for p in a.pages[s]:
                held[p] += 1
        assert held == a.holders.tolist()
        assert sorted(a.free_pages) == [p for p in range(n_pages) if held[p] == 0]


def test_refusals():
    a = PageAllocator(4, 8)
    s = a.add()
    with pytest.raises(ValueError):
        PageAllocator(0, 8)
    with pytest.raises(ValueError):
        a.extend([s, s], [1, 1])
    with pytest.raises(ValueError):
        a.extend([s], [-1])
    with pytest.raises(ValueError):
        a.extend([s], [1, 2])
    with pytest.raises(ValueError):
        a.truncate(s, 1)
    with pytest.raises(OutOfPages):
        a.extend([s], [33])
    with pytest.raises(KeyError):
        a.fork(99)
    assert a.extend([s], [32]) == [] and len(a.pages[s]) == 4 and not a.free_pages


def test_reserved_pages_are_not_shared():
    a = PageAllocator(4, 8)
    s = a.add()
    a.extend([s], [9])                 # two pages reserved, nothing cached in the second
    a.length[s] = 8
    t = a.fork(s)
    assert a.pages[t] == a.pages[s][:1]
    assert a.extend([s, t], [1, 1]) == [] and a.pages[s][1] != a.pages[t][1]
