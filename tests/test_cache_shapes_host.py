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


#: calls whose batch is taken in several launches: dim, B, n, heads, group, prefix, own tokens, and the launches
LAUNCHES = [(64, 1501, 2, 4, 1, 1000, 5, 2), (8, 3001, 1, 4, 2, 333, 5, 4), (40, 2001, 1, 3, 3, 700, 3, 2), (128, 3001, 1, 4, 2, 1000, 5, 2),
            (256, 1501, 1, 3, 4, 600, 33, 2)]
#: and where the rows of all sequences over the prefix are in tiles of 32: dim, B, n, heads, group, prefix, own tokens, types
TWO_TILES = [(64, 16, 45, 5, 1, 16150, 90, (0, 1)), (64, 16, 21, 5, 1, 9001, 33, (0, 1)), (64, 16, 11, 5, 2, 9001, 33, (0, 1)),
             (128, 16, 11, 5, 2, 6001, 33, (1,)), (128, 32, 7, 3, 3, 6001, 20, (1,)), (128, 32, 7, 3, 3, 6001, 0, (1,))]


def test_batches_in_several_launches(run):  # noqa: F811
    run(CALLS + f"shapes = {LAUNCHES!r}" + r'''
for dim, B, n, heads, group, P_, L_, launches in shapes:
    h, _ = plan(heads, dim, 4, 64)
    for precision in (0, 1):
        rc, made = shared(h, B, n, heads * group, P_, L_, precision=precision)
        assert rc == 0 and len(made) == 2 * launches, (dim, B, len(made))       # each with its join
        assert B % launches                                                     # and the last takes fewer
    L.wf_cache_destroy(h)
''')


def test_prefixes_in_tiles_of_32_rows(run):  # noqa: F811
    run(CALLS + f"shapes = {TWO_TILES!r}" + r'''
for dim, B, n, heads, group, P_, L_, precisions in shapes:
    h, _ = plan(heads, dim, 4, 64)
    for precision in precisions:
        rc, made = shared(h, B, n, heads * group, P_, L_, precision=precision)
        each = n * group
        # a launch and its join, of four waves for two tiles of 16; of whole splits of the tiles of all
        # rows and of each sequence's, and no multiple of each sequence's alone
        assert rc == 0 and len(made) == 2 and made[0].block == 256, (dim, B, n)
        first, own = heads * -(-B * each // 32), B * heads * -(-each // 32) if L_ else 0
        assert made[0].grid > own and (made[0].grid - own) % first == 0 and not (own and made[0].grid % own == 0), (dim, B, n, made[0].grid)
    L.wf_cache_destroy(h)
''')
