"""What calls of a decoder's cache launch, on the CPU: batches of prompts and steps together are within a launch's limits
however long the prompts are, and the calls of the GPU tests take the paths that they are there for."""
import pytest

import cache_plan as plan
from test_gpu_cache_mixed import MIXED
from test_gpu_cache_order import PROMPTS, STEPS, said

ITEMS, GRID = 2 ** 23 - 1, 65535


@pytest.mark.parametrize("n_seq,prompt,nh,nkv,hd", [
    (256, 131072, 32, 8, 128), (2049, 32768, 32, 8, 128), (2, 2 ** 30, 32, 8, 128), (65536, 65536, 12, 12, 64), (1, 2 ** 31 - 256, 16, 4, 64), (4096, 8192, 64, 1, 64)])
def test_one_prompt_beside_steps(n_seq, prompt, nh, nkv, hd):
    for causal in (True, False):
        p = plan.attention(n_seq - 1 + prompt, n_seq, prompt, prompt, nh, nkv, hd, causal)
        assert p.fits and p.prompt and p.tiles > 0
        assert n_seq * nkv * p.tiles * p.splits <= ITEMS and p.tiles * p.splits <= GRID
        assert p.tiles * p.tile_rows <= prompt * (nh // nkv) + p.tile_rows - 1


@pytest.mark.parametrize("n_seq,prompt,nh,nkv,hd", [
    (256, 131072, 32, 8, 128), (2049, 32768, 32, 8, 128), (2, 2 ** 30, 32, 8, 128), (65536, 65536, 12, 12, 64),
    (1, 2 ** 31 - 256, 16, 4, 64), (4096, 8192, 64, 1, 64)])
@pytest.mark.parametrize("kind,rot,queries", [(0, 0, True), (1, 64, True), (2, 18, True), (0, 0, False)])
def test_one_prompt_beside_steps_is_appended(n_seq, prompt, nh, nkv, hd, kind, rot, queries):
    p = plan.append(n_seq - 1 + prompt, n_seq, prompt, nh, nkv, hd, kind, rot, queries)
    assert p.fits and not p.step and p.vec == (rot != 18) and 0 < p.groups <= min(GRID, (prompt + 30) // 16)
    assert n_seq * p.parts * p.groups <= ITEMS
    v_parts = -(-p.v_columns // p.v_per)
    assert p.parts == p.q_parts + p.k_parts + v_parts and max(p.per, p.v_per) <= 256
    for columns, parts, per in ((p.q_columns, p.q_parts, p.per), (p.k_columns, p.k_parts, p.per), (p.v_columns, v_parts, p.v_per)):
        assert (parts - 1) * per < columns <= parts * per


def test_a_launch_of_fewer_groups_than_a_sequence_has():
    n, _, prompt, nh, nkv, hd = MIXED[0]
    p = plan.append(n - 1 + prompt, n, prompt, nh, nkv, hd, 1, hd)
    assert p.fits and 1 < p.groups < prompt // 16


def test_more_sequences_than_a_launch_takes():
    assert plan.append(2 ** 22, 2 ** 22, 1, 1, 1, 16).fits == 0  # 3 workgroups each
    assert plan.append(2 ** 21, 2 ** 21, 1, 1, 1, 16).fits == 1


@pytest.mark.parametrize("n,at,prompt,nh,nkv,hd", MIXED)
def test_mixed_batches_have_more_tiles_than_workgroups(n, at, prompt, nh, nkv, hd):
    p = plan.attention(n - 1 + prompt, n, prompt, prompt, nh, nkv, hd)
    tiles = -(-prompt * (nh // nkv) // p.tile_rows)
    assert p.prompt and p.by_length == (n <= 256) and p.splits == 1 and 1 < p.tiles < tiles and n * nkv * tiles > ITEMS


def test_what_fits_has_a_workgroup_for_every_tile():
    p = plan.attention(16 * 300, 16, 512, 2560, 12, 12, 64)
    assert p.fits and p.tiles == 512 // p.tile_rows


def test_one_tile_a_sequence_does_not_fit():
    assert plan.attention(2 ** 20, 2 ** 20, 1, 64, 8, 8, 64).fits == 0  # 2^23 tiles
    assert plan.attention(2 ** 20, 2 ** 20 - 1, 1, 64, 8, 8, 64).fits == 1


@pytest.mark.parametrize("name", [*PROMPTS, *STEPS])
@pytest.mark.parametrize("causal", [True, False])
def test_what_is_to_be_in_order_is(name, causal):
    case = {**PROMPTS, **STEPS}[name]
    p = plan.attention(*said(case), causal)
    assert p.fits and p.by_length and p.prompt == (name in PROMPTS)
    assert (p.splits > 1) == ("parts" in name or name in STEPS)
    if name in STEPS:
        assert p.tiles == int(name[name.index("of") + 3])
    (news, _), nh, nkv, *_ = case
    assert ("more tokens" in name) == (max(news) * (nh // nkv) > p.tiles * p.tile_rows)


def test_the_paths_of_the_order_tests_cover_both_tables_of_lengths():
    n = [len(case[0][0]) for case in PROMPTS.values()], [len(case[0][0]) for case in STEPS.values()]
    assert all(min(c) <= 64 < max(c) <= 256 for c in n) and max(n[0]) == 256
    rows = {plan.attention(*said(case)).tile_rows for case in PROMPTS.values()}
    assert rows == {64, 128}


def test_forms_of_the_bar_tests():
    p = plan.attention(9, 4, 5, 256, 8, 2, 64)
    assert not p.prompt and p.splits == 1
    for hd in range(16, 129, 16):
        assert plan.attention(238 * 6, 30, 130, 200, 12, 6, hd).prompt
