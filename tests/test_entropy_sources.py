"""Cross entropy: what its results do not show, from its sources (no GPU needed)."""
import re

from test_more_head_sources import kernels, source


def test_one_block_joins_a_tile_that_workers_share():
    """entropy_join has a block to each worker; of those that look at one tile exactly one may write it, and only where several had a part."""
    body = kernels(source("entropy.cu"))["entropy_join"][1]
    given_up = re.search(r"if \((.*)\) return;", body).group(1)
    given_up = re.sub(r"\(([^()?]*) \? ([^:]*) : ([^()]*)\)", r"((\2) if (\1) else (\3))", given_up)
    given_up = given_up.replace("||", "or").replace("(int)blockIdx.x", "block").replace("e.line.inner", "inner")
    stops = eval("lambda block, w0, w1, begin, tile, inner: " + given_up)
    for outer in (1, 2, 3, 8, 29):
        for inner in (1, 2, 3, 7, 32, 70):
            tiles = outer * inner
            for workers in {1, 2, 3, outer, 2 * outer, 5 * outer, 40, 148} - {0}:
                if workers > tiles:
                    continue
                begins = [tiles * w // workers for w in range(workers + 1)]
                worker_of = [((t + 1) * workers - 1) // tiles for t in range(tiles)]
                assert all(begins[w] <= t < begins[w + 1] for t, w in enumerate(worker_of))
                joined = []
                for block in range(workers):
                    tile = begins[block] // inner
                    w0, w1 = worker_of[tile * inner], worker_of[tile * inner + inner - 1]
                    if not stops(block, w0, w1, begins[block], tile, inner):
                        joined.append(tile)
                shared = [t for t in range(outer) if worker_of[t * inner] != worker_of[t * inner + inner - 1]]
                assert joined == shared, (outer, inner, workers)
