"""Cross entropy: what its results do not show, from its sources (no GPU needed)."""
import re

import pytest

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


# ---------------------------------------------------------------------------------------------- what goes before the wait of an early start
WAIT = "ep_wait_for_launch_before()"
TOUCHES = re.compile(r"\b(?:load_|store_|ld_|st_|tma_|bulk_|copy_|copies_|atomic|__ld|__st|ask_|target_of|memcpy|memset)\w*\s*\(")


def parameters(head):
    """(pointers, structs) among a kernel's parameters, by name."""
    depth, part, parts = 0, "", []
    for c in head[head.index("(", head.index(" void ")) + 1:head.rindex(")")]:
        depth += (c in "(<[") - (c in ")>]")
        if c == "," and depth == 0:
            parts.append(part)
            part = ""
        else:
            part += c
    pointers, structs = set(), set()
    for p in parts + [part]:
        name = re.search(r"(\w+)\s*$", p).group(1)
        kind = p[:p.rindex(name)]
        if "*" in kind:
            pointers.add(name)
        elif not re.search(r"\b(?:int|float|double|bool|unsigned|int32_t|int64_t|uint32_t|CUtensorMap)\b", kind):
            structs.add(name)
    return pointers, structs


def ways_to_the_wait(body):
    """The text ahead of each wait; a block that has a wait of its own (and leaves) is one way, what is around it another."""
    ways = []
    while WAIT in body:
        at = body.index(WAIT)
        ways.append(body[:at])
        open_at = []
        for i, c in enumerate(body[:at]):
            if c == "{":
                open_at.append(i)
            elif c == "}":
                open_at.pop()
        if len(open_at) < 2:      # (the first is the body's own)
            return ways
        start, depth, end = open_at[1], 0, len(body)
        for i in range(start, len(body)):
            depth += (body[i] == "{") - (body[i] == "}")
            if depth == 0:
                end = i + 1
                break
        body = body[:start] + ";" + body[end:]
    return []


def touched_before_the_wait(head, body):
    """What a kernel does ahead of its wait that may be a read or a write of global memory."""
    ways, found = ways_to_the_wait(body), []
    if not ways:
        return ["no wait"]
    pointers, structs = parameters(head)
    for before in ways:
        found += [m.group(0) for m in TOUCHES.finditer(before)]
        for name in pointers:   # any use at all, but for a comparison with nothing
            found += [name] * len(re.findall(r"(?<![\w.>])%s\b(?!\s*[!=]=\s*(?:nullptr|NULL))" % name, before))
        for name in structs:    # a member that is read through or handed on
            member = r"(?<![\w.>])%s(?:\.\w+)+" % name
            found += re.findall(member + r"\s*(?:\[|->)", before) + re.findall(r"(?<=[(,=!&|])\s*\*\s*" + member, before)
            found += re.findall(r"\w+\s*\([^;{}]*?\b%s\s*[,)]" % name, before)
    return found


@pytest.mark.parametrize("name,least", [("entropy.cu", 9), ("experts.cu", 5), ("linear.cu", 2), ("norm.cu", 1), ("route.cu", 1)])
def test_nothing_is_touched_before_the_wait(name, least):
    known = kernels(source(name))
    waiting = [k for k, (head, body) in known.items() if WAIT in body]
    assert len(waiting) >= least, waiting
    for kernel in waiting:
        assert touched_before_the_wait(*known[kernel]) == [], kernel


@pytest.mark.parametrize("early,line", [
    (True, "const float v = x[threadIdx.x];"), (True, "*out = 1.f;"), (True, "const float v = *x;"), (True, "const float b = load_param(x, 0, 1);"),
    (True, "if (*w.scale) return;"), (True, "w.rows.g[3] = 0.f;"), (True, "helper(w, 3);"), (True, "use(out);"), (True, "const int k = w.plan->groups;"),
    (False, "const int i = blockIdx.x * n + w.count;"), (False, "__shared__ float part[8]; part[0] = 0.f;"), (False, "if (out == nullptr) return;"),
    (False, "const int a = 2 * w.count;")])
def test_the_check_tells_a_read_before_the_wait(early, line):
    text = """
template <typename T>
__global__ void __launch_bounds__(256) some_kernel(const T *x, const Work w, int n, float *out) {
    const int lane = threadIdx.x & 31;
    %s
    ep_wait_for_launch_before();
    out[lane] = x[lane] + w.rows.g[n];
}
"""
    assert bool(touched_before_the_wait(*kernels(text % line)["some_kernel"])) == early
    late = (text % "").replace("    out[lane]", "    %s\n    out[lane]" % line)
    assert touched_before_the_wait(*kernels(late)["some_kernel"]) == []
    assert touched_before_the_wait(*kernels(late.replace("ep_wait_for_launch_before();", ""))["some_kernel"]) == ["no wait"]


def test_the_check_follows_either_branch():
    text = """
__global__ void two_ways(const float *x, int n, float *out) {
    if (n > 3) {
        %s
        ep_wait_for_launch_before();
        out[0] = x[0];
        return;
    }
    %s
    ep_wait_for_launch_before();
    out[1] = x[1];
}
"""
    for first, second, touched in (("", "", False), ("out[2] = 0.f;", "", True), ("", "out[2] = 0.f;", True)):
        assert bool(touched_before_the_wait(*kernels(text % (first, second))["two_ways"])) == touched
    only_one = text.replace("    %s\n    ep_wait_for_launch_before();\n    out[1]", "    out[1]") % ""
    assert touched_before_the_wait(*kernels(only_one)["two_ways"]) == ["no wait"]
