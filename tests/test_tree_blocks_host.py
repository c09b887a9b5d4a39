"""What a tree refuses before it looks at a GPU."""
import pytest


def test_sizes_of_a_tree_are_refused():
    import paper_2607_01308_gb300 as cm
    for nodes, freed in ((0, None), (257, None), (8, -1), (8, 1 << 31)):
        with pytest.raises(ValueError):
            cm.QTree(None, nodes, max_freed=freed)
