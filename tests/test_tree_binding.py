"""What Context.spd_tree_plan hands out, without a GPU: the library's call is only looked at."""
import torch

import paper_2409_19134_amd as spd
from paper_2409_19134_amd import binding as b
from test_tree_host import _Stream, _context, _here


class Lib:
    def spd_tree_plan(self, ctx, n_users, n_new, parents, first, words, seen, depth, positions, stream):
        self.first, self.positions = first, positions
        return spd.SPD_OK


class Parents:
    """A tensor that says it is on the context's device, and makes others beside it that say so too."""

    def __new__(cls, t, monkeypatch):
        made = b.Tree.__init__

        def init(self, n_tokens, words=1, device=None):
            made(self, n_tokens, words, "cpu")
            for name in ("seen", "depth", "positions"):
                setattr(self, name, _here(getattr(self, name)))

        monkeypatch.setattr(b.Tree, "__init__", init)
        return _here(t)


def test_positions_are_handed_out_only_where_they_were_made(monkeypatch):
    lib = Lib()
    monkeypatch.setattr(b, "lib", lib)
    parents = Parents(torch.zeros(3, dtype=torch.int32), monkeypatch)
    tree = _context().spd_tree_plan(parents, [1, 2], stream=_Stream)
    assert tree.positions is None and lib.first is None and lib.positions is None
    tree = _context().spd_tree_plan(parents, [1, 2], first=[5, 6], stream=_Stream)
    assert tree.positions is not None and lib.positions == tree.positions.data_ptr()
    # one of the caller's keeps what it has
    kept = tree.positions
    assert _context().spd_tree_plan(parents, [1, 2], tree=tree, stream=_Stream) is tree
    assert tree.positions is kept and lib.positions is None
