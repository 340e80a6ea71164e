"""Which kernels the windowed and the shared attention launch for which calls, on
stand-ins for the HIP calls (no GPU needed): what other tests and figures rely on."""
from paper_2607_19082_amd import wf  # noqa: F401 (built by the fixture below)
from test_cache_host import run  # noqa: F401 (a fixture)
from test_cache_runs_host import CALLS


def test_sequences_are_not_a_die_each(run):  # noqa: F811
    """A wave or two take a tile of rows: the launch is 8 times whole workgroups of
    a die's tiles where work is dealt to dies, and whole workgroups of all where it
    is not.  Sequences of one head may be of unequal lengths, so they are dealt only
    with 8 heads, or 16."""
    run(CALLS + r'''
tiles = 257                                             # of 32 rows, a sequence and head
for heads, B in ((1, 8), (2, 8), (4, 6), (2, 4), (8, 3), (16, 2), (3, 5)):
    h, _ = plan(heads, 64, 4, 1024)
    rc, made = window(h, B, 32 * tiles, heads, 9000, 5, 0)
    assert rc == 0 and len(made) == 1 and made[0].block == 256
    units, grids = B * heads, {}
    for teams in (4, 2):
        grids[8 * -(-units // 8 * tiles // teams) if heads % 8 == 0 else -(-units * tiles // teams)] = teams
    assert made[0].grid in grids, (heads, B, made[0].grid, grids)
    if units % 8 == 0 and heads % 8:                    # (the two ways differ here)
        assert made[0].grid != 8 * -(-units // 8 * tiles // grids[made[0].grid])
''')
