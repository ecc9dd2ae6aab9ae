"""The rule by which a block of the token kernel leaves values out of the search for its
best, under any order of its warps' steps (no GPU): a model of the rule, not the kernel."""
import random


def best_of_block(rng, z, warps, lanes, top, own_words):
    """The candidates' best of z (one value a lane and step), warps taking turns at random
    after the first step's barrier.  A warp's step: read what all warps say (the live bound,
    `at or above`), offer, say its own candidates' bound; after the first step a bound that
    later values have to be above: from words of the first step, or (own_words False) from
    the live ones as they were read."""
    steps = -(-len(z) // (warps * lanes))
    each = -(-top // warps)

    def values(w, s):
        first = (s * warps + w) * lanes
        return [(z[i], i) for i in range(first, min(first + lanes, len(z)))]

    def bound_of(candidates):
        kept = sorted((v for v, _ in candidates), reverse=True)
        return kept[each - 1] if len(kept) >= each else -1

    said = [bound_of(values(w, 0)) for w in range(warps)]
    first = min(said)
    strict, found, at, floor = [-1] * warps, [[] for _ in range(warps)], [0] * warps, [None] * warps
    while any(s < steps for s in at):
        w = rng.choice([w for w in range(warps) if at[w] < steps])
        if floor[w] is None:
            floor[w] = min(said)
            continue
        found[w] += [(v, i) for v, i in values(w, at[w]) if v > strict[w] and v >= floor[w]]
        said[w] = max(said[w], bound_of(found[w]))
        if at[w] == 0:
            strict[w] = max(strict[w], first if own_words else floor[w])
        at[w], floor[w] = at[w] + 1, None
    best = sorted((c for f in found for c in f), key=lambda c: (-c[0], c[1]))
    return [i for _, i in best[:top]]


def wrong(own_words, trials=4000):
    rng = random.Random(5)
    n = 0
    for _ in range(trials):
        warps, lanes, top = rng.choice((2, 3, 4)), rng.choice((1, 2, 4)), rng.randint(1, 5)
        z = [rng.randint(0, rng.choice((1, 2, 9))) for _ in range(rng.randint(max(top, warps * lanes), 6 * warps * lanes))]
        want = sorted(range(len(z)), key=lambda i: (-z[i], i))[:top]
        n += best_of_block(rng, z, warps, lanes, top, own_words) != want
    return n


def test_ties_go_to_the_lowest_index_in_any_order_of_the_warps():
    assert wrong(True) == 0


def test_a_bound_read_from_the_live_words_would_lose_ties():
    """The model does see what the first step's own words are for."""
    assert wrong(False) > 0
