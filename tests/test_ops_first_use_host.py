"""First use from several threads: the table of entries that calls look into is never
empty once an object exists.  CPU only."""

from paper_2606_19163_amd import ops

from test_ops_host import built  # noqa: F401  (builds the library)


class Watched:
    """The library, which looks at the table at every step of the binding."""

    def __init__(self, lib, seen):
        self.lib, self.seen = lib, seen

    def _look(self, entry):
        self.seen.append(sorted(ops._fast))
        return entry

    def __getattr__(self, name):
        return self._look(getattr(self.lib, name))

    def __getitem__(self, name):
        return self._look(self.lib[name])


def test_a_second_binding_leaves_the_table_whole(monkeypatch):
    """A thread that found the library unbound binds it again, while another one,
    which was faster, makes its calls."""
    real = ops.lib()
    whole = sorted(ops._fast)
    assert len(whole) == 12
    seen = []
    monkeypatch.setattr(ops, "_bound", None)
    monkeypatch.setattr(ops, "_lib", lambda: Watched(real, seen))
    ops.lib()
    assert seen and all(names == whole for names in seen)
    assert sorted(ops._fast) == whole


def test_the_table_is_there_before_the_library_counts_as_bound(monkeypatch):
    real, seen = ops.lib(), []
    monkeypatch.setattr(ops, "_bound", None)
    monkeypatch.setattr(ops, "_fast", {})
    monkeypatch.setattr(ops, "_lib", lambda: Watched(real, seen))
    ops.lib()
    assert not any(seen) and len(ops._fast) == 12
