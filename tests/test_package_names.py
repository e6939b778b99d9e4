"""Every name that the package's functions look up globally exists (no GPU needed)."""
import builtins
import dis
import importlib
import types

import pytest


def codes(code):
    yield code
    for c in code.co_consts:
        if isinstance(c, types.CodeType):
            yield from codes(c)


@pytest.mark.parametrize("name", ["binding", "build"])
def test_global_names_exist(name):
    module = importlib.import_module("paper_2604_01000_b200." + name)
    code = compile(open(module.__file__).read(), module.__file__, "exec")
    missing = {(c.co_name, i.argval) for c in codes(code) for i in dis.get_instructions(c)
               if i.opname == "LOAD_GLOBAL" and not hasattr(module, i.argval) and not hasattr(builtins, i.argval)}
    assert not missing
