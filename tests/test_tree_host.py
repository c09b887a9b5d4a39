"""The operators around a tree of drafted tokens where no GPU is needed: missing contexts are refused, the descriptors are laid
out as a C compiler lays them out, the test reference's walk draws the target's distribution."""
import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import tree_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_null_arguments_are_refused():
    import paper_2607_01308_gb300 as cm
    bad = cm.Status.ERR_INVALID_ARG
    assert cm.lib.cm_qcache_tree(None, None, None, None, 0, 1, None, None, None) == bad
    assert cm.lib.cm_qk_rotate(None, None, None) == bad
    assert cm.lib.cm_qcache_attend_tree(None, None, 0, None, None, None, 1, None, 0, None) == bad
    assert cm.lib.cm_tree_verify(None, None, None) == bad
    assert cm.lib.cm_qcache_keep(None, None, None, None, None, None, 0, None, None, 0, None, None) == bad
    assert "context" in cm.cm_last_error_message()


def test_structs_are_laid_out_as_in_c(tmp_path):
    import paper_2607_01308_gb300 as cm
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = ("cm_qk_rows", "cm_tree_drafts")
    fields = [(s, f[0]) for s in structs for f in getattr(cm, s)._fields_]
    body = "".join('printf("%%zu\\n", sizeof(%s));\n' % s for s in structs)
    body += "".join('printf("%%zu\\n", offsetof(%s, %s));\n' % f for f in fields)
    path, exe = str(tmp_path / "x.c"), str(tmp_path / "x")
    with open(path, "w") as f:
        f.write("#include <stddef.h>\n#include <stdio.h>\n#include \"cm.h\"\nint main(void) {\n%sreturn 0;\n}\n" % body)
    subprocess.run([cc, "-std=c11", "-Wall", "-Werror", "-I" + os.path.join(ROOT, "include"), path, "-o", exe], check=True)
    got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    want = [ctypes.sizeof(getattr(cm, s)) for s in structs] + [getattr(getattr(cm, s), f).offset for s, f in fields]
    assert got == want
    from paper_2607_01308_gb300 import tree
    assert len(tree._pack_rows(*[0] * 16, *[0] * 3, 0.0, 0)) == ctypes.sizeof(cm.cm_qk_rows)
    assert len(tree._pack_drafts(*[0] * 17)) == ctypes.sizeof(cm.cm_tree_drafts)


@pytest.mark.parametrize("drawn", [True, False])
def test_the_walk_draws_the_targets_distribution(drawn):
    """The first token behind the root (the accepted row's or the chosen one) over many random numbers: each frequency within
    five standard deviations, sqrt(p (1 - p) / n)."""
    rng = np.random.default_rng(1)
    vocab, fan, n = 6, 3, 20000
    p, q = (x / x.sum() for x in (rng.random(vocab) ** 2, rng.random(vocab)))
    target = np.tile(p.astype(np.float32), (fan + 1, 1))
    draft = np.tile(q.astype(np.float32), (fan + 1, 1)) if drawn else None
    counts = np.zeros(vocab)
    for _ in range(n):
        tokens = [0] + (rng.choice(vocab, fan, p=q).tolist() if drawn else [4, 1, 1])
        path, kept, chosen = ref.verify([0, fan + 1], [-1, 0, 0, 0], tokens, target, draft, rng.random(fan + 1, dtype=np.float32),
                                        rng.random(1, dtype=np.float32), 256)
        counts[tokens[path[1]] if kept[0] > 1 else chosen[0]] += 1
    assert np.all(np.abs(counts / n - p) <= 5 * np.sqrt(p * (1 - p) / n))


def test_reference_masks():
    masks, positions = ref.plan([0, 4, 4, 6], [10, 0, -3], [-1, 0, 0, 2, -1, 7], 7, 1)
    assert masks == [1, 3, 5, 13, 1, 2, None] and positions == [10, 11, 11, 12, 0, 0, None]
    masks, positions = ref.plan([0, 3], [5], None, 3, 1)
    assert masks == [1, 3, 7] and positions == [5, 6, 7]
