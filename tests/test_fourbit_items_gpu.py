"""Attention over the cache of 4 bits where a block's items alternate between two row tiles and one: chunks of prompts among short
ones, all of them so short that an item is soon over and the next one's queries are already there."""
import random

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from test_fourbit_attention_gpu import _build, _check, _run  # noqa: E402


def _some(s, every):
    """The same call, of which every so many sequences are checked."""
    return dict(s, news=[n if b % every == 0 else 0 for b, n in enumerate(s["news"])])


def _news(kind, B, seed):
    """Rows of each sequence at 4 heads a key head, whose row tiles have 32 of them: 33 to 64 are an item of two."""
    rng = random.Random(seed)
    if kind == "alternating":  # each key head: an item of two row tiles, then one of one
        return [3, 3, 1] + [rng.randint(65, 90) for _ in range(B - 3)]
    if kind == "three apart":  # an odd number of items of one row tile in a row
        return [2] + [64, 5, 40] * (B // 3)
    return [rng.choice([1, 7, 31, 33, 50, 64, 70, 110, 128]) for _ in range(B)]


@pytest.mark.parametrize("kind", ["alternating", "three apart", "any"])
@pytest.mark.parametrize("d,kvh", [(128, 8), (128, 1), (64, 8), (64, 3)])
def test_items_of_two_row_tiles_and_of_one(kind, d, kvh):
    """At most 128 keys: a single key tile, of which an item of one row tile has nothing for the second slot."""
    news = _news(kind, 240, d + kvh)
    lens = [max(n, min(128, n + b % 60)) for b, n in enumerate(news)]
    s = _build(lens, news, 4 * kvh, kvh, d, 32, torch.bfloat16 if kvh != 3 else torch.float16, seed=kvh)
    want = _run(s)
    _check(_some(s, 6), want)
    for _ in range(40):
        assert torch.equal(_run(s), want)


@pytest.mark.parametrize("d", [64, 128])
def test_the_same_with_contexts_of_several_key_tiles(d):
    news = _news("any", 150, d)
    lens = [n + 37 * b % 500 for b, n in enumerate(news)]
    s = _build(lens, news, 8, 2, d, 64, torch.bfloat16, seed=d)
    want = _run(s)
    _check(_some(s, 4), want)
    for _ in range(20):
        assert torch.equal(_run(s), want)


@pytest.mark.parametrize("n", [2, 17, 40])
@pytest.mark.parametrize("d", [64, 128])
def test_key_tiles_that_are_zeros_between_others(d, n):
    """Tiles of which no block is in the pool (nothing is copied for them, so they are complete as soon as their zeros are written)
    and tiles of which some are, in the stages where other tiles' codes have been; values far from zero."""
    bs, B = 16, 24
    lens = [n + 90 * b % 1500 + 200 for b in range(B)]
    s = _build(lens, [n] * B, 8, 2, d, bs, torch.bfloat16, vs=50.0, seed=n)
    zero = torch.zeros(1, *s["cache"].shape[1:], dtype=torch.uint8, device="cuda")
    at = torch.cat([s["cache"], zero]), s["cache"].shape[0]
    for b in range(B):
        used = (lens[b] + bs - 1) // bs
        for j in range(used):
            if j // 8 % 3 == 1 or j % 5 == b % 5:  # every third tile of 128 keys, and some blocks of the others
                s["table"][b, j] = (-1, at[1], 2 ** 31 - 1)[j % 3]
                s["slots"][b][j * bs:(j + 1) * bs] = at[1] * bs + torch.arange(bs, device="cuda")[:lens[b] - j * bs]
    want = _run(s)
    _check(dict(s, cache=at[0]), want)
    for _ in range(20):
        assert torch.equal(_run(s), want)
