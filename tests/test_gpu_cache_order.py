"""cache_attention where sequences are taken in order of the keys that they see: prompts of up to 256 sequences, and steps
of several tiles a sequence, some with more tokens than was said. test_cache_plan_host.py checks on the CPU that these
calls take that order. Results are held to the bars of test_gpu_cache.py."""
import numpy as np
import pytest

from test_gpu_cache import Batch, run_attend

pytestmark = pytest.mark.gpu


def ragged(n, new, behind, seed, far=0):
    """Tokens and cached ones of n sequences: few of each as a rule, the most once (`far` cached ones
    more); some idle."""
    rng = np.random.default_rng([n, new, behind, seed])
    news = [int(v) for v in np.minimum(rng.geometric(4 / (new + 3), n), new)]
    lens = [max(0, k + int(b)) for k, b in zip(news, rng.integers(-3, behind + 1, n))]
    news[n // 2], lens[n // 2] = new, new + behind + far
    news[n // 3], lens[n // 3] = 0, 40
    return news, lens


# name: tokens and lengths, query and key heads, features of a head, the longest numbers that are said (0: as they are)
PROMPTS = {
    "65 sequences": (ragged(65, 90, 100, 1), 12, 12, 64, 0, 0),
    "66, wide heads": (ragged(66, 70, 300, 2), 16, 8, 128, 0, 0),
    "200, one key head": (ragged(200, 90, 60, 3), 6, 1, 80, 0, 0),
    "256": (ragged(256, 40, 50, 4), 4, 2, 32, 0, 0),
    "256, more tokens than said": (ragged(256, 100, 50, 5), 4, 4, 64, 40, 80),
    "130, many tiles": (ragged(130, 400, 30, 6), 3, 3, 16, 0, 0),
    "8, heads of 64": (([100, 0, 7, 64, 65, 130, 1, 33], [100, 50, 300, 64, 1000, 140, 0, 33]), 96, 96, 64, 0, 0),
    "8, heads of 128": (([100, 0, 7, 64, 65, 130, 1, 33], [100, 50, 300, 64, 1000, 140, 0, 33]), 64, 64, 128, 0, 0),
    "5, heads of 64": (([128, 128, 3, 128, 60], [128, 700, 3, 700, 2]), 80, 80, 64, 0, 0),
    "70, in parts": (ragged(70, 50, 2300, 7), 2, 2, 64, 0, 0),
}
STEPS = {
    "8 of 2 tiles": (ragged(8, 8, 300, 8), 32, 8, 64, 0, 2 ** 15),
    "12 of 4 tiles": (ragged(12, 8, 700, 9, 9000), 64, 8, 128, 0, 12000),
    "90 of 2 tiles": (ragged(90, 5, 200, 10), 8, 2, 64, 0, 2 ** 14),
    "128 of 3 tiles in one head": (ragged(128, 3, 100, 11), 16, 1, 96, 0, 2 ** 14),
    "40 of 2 tiles, more tokens than said": (ragged(40, 30, 400, 12), 12, 3, 48, 5, 2 ** 16),
    "7 of 3 tiles, more tokens than said": (ragged(7, 130, 900, 13, 30000), 6, 2, 80, 11, 2 ** 18),
}


def said(case):
    """m_tokens, n_seq, max_new, max_len and the heads of a case's call."""
    (news, lens), nh, nkv, hd, new, length = case
    return sum(news), len(news), new or max(news), length or max(lens), nh, nkv, hd


@pytest.mark.parametrize("name", [*PROMPTS, *STEPS])
@pytest.mark.parametrize("causal", [True, False])
def test_order(hip, name, causal):
    case = {**PROMPTS, **STEPS}[name]
    (news, lens), nh, nkv, hd, _, _ = case
    rng = np.random.default_rng(len(name))
    b = Batch(hip, rng, news, lens, 16, nkv, hd, holes="many" in name)
    _, _, b.most_new, b.longest, *_ = said(case)
    print(f"attention in order: {name}, causal={causal}", flush=True)
    run_attend(hip, rng, b, nh, causal=causal)
    path = hip.last_path()
    assert path.startswith(f"cache {'prompt' if name in PROMPTS else 'split'} {hd},")
    run_attend(hip, rng, b, nh, kind="i8", causal=causal)
