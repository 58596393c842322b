"""The grouped products take every call that a form of theirs has a grid for, and launch every workgroup that the form needs; the adapters launch every
tile of the height and every part of K that they take.  Launches are written down instead of going out; no GPU."""
import pytest

from test_groups_launch_sizes import most_tiles, run  # noqa: F401  (a fixture)
from test_kv4_launch_sizes import fits, workgroups

OPS = ["e0m4_matmul_grouped", "e0m8_matmul_grouped", "e0m4_bf16_matmul_grouped"]
# rows of a tile, columns and threads of a workgroup
FORMS = {1: (16, 64, 256), 2: (16, 32, 256), 3: (32, 64, 256), 4: (128, 256, 256), 5: (64, 128, 512), 6: (128, 128, 256)}


def column_blocks(call, columns):
    return -(-(call["N"] // 2) // (columns // 2)) if call["gated"] else -(-call["N"] // columns)


def room(rows, groups, height):
    """Tiles that a launch has room for: whole ones, and one for each group."""
    return rows // height + min(rows, groups)


def work_items(call, form):
    """Of a launch, without what rounds it up (at most four workgroups for each of eight parts of the chip)."""
    height, columns, threads = FORMS[form]
    return room(call["rows"], call["groups"], height) * column_blocks(call, columns) * threads


@pytest.mark.parametrize("op", OPS)
def test_calls_that_some_form_has_a_grid_for_are_taken(run, op):  # noqa: F811
    least = 64 if op == "e0m8_matmul_grouped" else 32
    sizes = [(64, 64, 1 << 24, least), (1000, 1023, 1 << 20, least), (1, 1, 1 << 24, least), (200, 200, 1 << 23, 64), (254, 1023, 1 << 24, 64), (256, 256, 1 << 24, 64), (257, 257, 1 << 24, 64),
             (1 << 24, 1023, 16384, 128), (1 << 24, 1, 1 << 15, 128), (1 << 24, 1, 1 << 16, 128), (1 << 20, 8, 1 << 19, 128), (40000, 1023, 1 << 22, 128)]
    calls = [dict(op=op, rows=rows, groups=groups, N=N, K=K, group=least, gated=gated) for rows, groups, N, K in sizes for gated in (0, 1)]
    calls = [c for c in calls if not (c["gated"] and c["N"] * c["K"] > 1 << 30)]       # (the gate's half of a buffer is at most 1 GiB)
    taken = refused = 0
    for call, (rc, launches) in zip(calls, run(calls)):
        least_items = min(work_items(call, f) for f in FORMS)
        if rc == 0:
            assert len(launches) == 1, call
            fits(launches[0])
            taken += 1
        else:
            assert rc == -2 and not launches and least_items > (1 << 32) - 64 * 256, call
            refused += 1
        # what the header says of the limit
        tiles, blocks = room(call["rows"], call["groups"], 128), -(-call["N"] // 256)
        assert tiles * blocks > (1 << 24) - 64 or rc == 0, call
    assert taken and refused


@pytest.mark.parametrize("form", sorted(FORMS))
@pytest.mark.parametrize("op", OPS)
def test_a_form_refuses_only_what_does_not_fit_its_own_grid(run, op, form):  # noqa: F811
    height, columns, threads = FORMS[form]
    calls = []
    for rows, groups in ((64, 64), (1000, 1023), (1 << 20, 16), (1 << 24, 1023)):
        tiles = room(rows, groups, height)
        for gated in (0, 1):
            most = ((1 << 32) - 1) // threads // tiles * columns
            for N in (most // 64 * 64 // 2, most // 64 * 64 - 64 * columns, most // 64 * 64 + 2 * columns):
                if 64 <= N <= 1 << 24:
                    calls.append(dict(op=op, rows=rows, groups=groups, N=N // 64 * 64, K=64, group=64, gated=gated, knobs={"grouped_form": form}))
    for call, (rc, launches) in zip(calls, run(calls)):
        items = work_items(call, form)
        if rc == 0:
            (grid, block, lds), = launches
            fits(launches[0])
            assert block[0] == threads and workgroups(launches[0]) >= most_tiles(call["rows"], call["groups"], height) * column_blocks(call, columns), call
        else:
            assert rc == -2 and not launches and items > (1 << 32) - 64 * threads, call


def test_adapters_launch_every_tile_and_part(run):  # noqa: F811
    """Rows of an adapter are counted as if all of them were in use, as the launch does."""
    calls = [dict(op="lora", rows=rows, groups=groups, rank=rank, N=N, K=K, dtype=dtype)
             for rows, groups, K in ((1, 1, 8), (1, 1023, 1 << 20), (16, 1, 1024), (17, 1, 1024), (64, 1, 4096), (65, 1, 4096), (1000, 2, 4096), (1 << 20, 1023, 512))
             for rank in (8, 32, 40, 64, 72, 128) for N in (8, 4096, 1 << 20) for dtype in (0, 1)]
    from paper_2403_20041_amd import binding

    for call, (rc, launches) in zip(calls, run(calls)):
        rows, groups, rank = call["rows"], call["groups"], call["rank"]
        each = rows // min(rows, groups)
        heights = 32 if each > 64 and 32 < rank <= 64 else 16, 32 if each > 16 else 16
        assert rc == 0 and len(launches) == 2, call
        # (a part of K leaves a slab of rows x rank sums)
        parts = binding.e0m4_lora_workspace_bytes(rows, groups, rank, call["N"], call["K"]) // (rows * rank * 4)
        assert parts >= 1 and workgroups(launches[0]) >= most_tiles(rows, groups, heights[0]) * parts, call
        for launch in launches:
            fits(launch)
        assert workgroups(launches[1]) >= most_tiles(rows, groups, heights[1]), call
