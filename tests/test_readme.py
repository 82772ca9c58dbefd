"""The steps over pages that the README shows, run against the binding's own signatures with calls that only note their arguments: what one
call gives back the others of the step must not need.  Needs no GPU."""
import inspect
import os
import re

from paper_2502_01941_amd import kv4

README = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")


class Value:
    """Anything that the text does not define; any attribute of it is another such thing, the same one every time."""

    def __init__(self, name):
        self._name, self._parts = name, {}

    def __getattr__(self, name):
        return self._parts.setdefault(name, Value(f"{self._name}.{name}"))


class Names(dict):
    def __missing__(self, name):
        return self.setdefault(name, Value(name))


def _steps():
    """The README's blocks of code in which the binding of the pages is called."""
    blocks, block = [], []
    for line in open(README).read().splitlines() + ["."]:
        if line.startswith("    ") or (block and not line.strip()):
            block.append(line[4:])
        elif block:
            blocks.append("\n".join(block))
            block = []
    return [b for b in blocks if "kv4." in b]


def _calls(code):
    """[(name, arguments by name)] of the calls in their order; arguments that the binding does not take raise."""
    made = []

    class Recorder:
        def __getattr__(self, name):
            real = getattr(kv4, name)
            if inspect.isclass(real):
                class Made(Value):
                    empty = staticmethod(lambda *a, **k: Value(name))

                    def __init__(self, *a, **k):
                        inspect.signature(real).bind(*a, **k)
                        super().__init__(name)
                return Made

            def call(*args, **kw):
                bound = inspect.signature(real).bind(*args, **kw)
                bound.apply_defaults()
                made.append((name, bound.arguments))
                return Value(name), Value(name)
            return call
    names = Names(kv4=Recorder())
    exec(re.sub(r"^from .* import kv4$", "", code, flags=re.M), {"__builtins__": {}}, names)
    return made


def test_the_steps_are_found():
    names = [name for code in _steps() for name, _ in _calls(code)]
    assert {"attention", "window_attention", "tree_attention", "tree_plan", "tree_keep", "pages_trim"} <= set(names)


def test_pages_are_given_back_only_where_no_call_reads_them():
    """A trim with a window takes the pages between sinks and window of the table: every attention over that table has that window or a
    shorter one, and those sinks or fewer."""
    trims = 0
    for code in _steps():
        calls = _calls(code)
        for name, trim in calls:
            if name != "pages_trim" or trim["window"] is None:
                continue
            trims += 1
            for what, read in calls:
                if "attention" not in what or read["block_table"] is not trim["block_table"]:
                    continue
                assert read.get("window") is not None and read["window"] <= trim["window"], what
                assert read["n_sinks"] <= trim["n_sinks"], what
    assert trims


def test_kept_drafts_go_by_the_plan():
    """A step that plans its trees gives their status to the call that keeps drafts."""
    for code in _steps():
        calls = _calls(code)
        if "tree_plan" in [name for name, _ in calls]:
            assert all(args["status"] is not None for name, args in calls if name == "tree_keep")
