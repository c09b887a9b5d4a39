"""The 8-bit cache's descriptors and calls from C: the layout that a C compiler gives them is that of the ctypes
mirrors, and the calls refuse a missing context. No GPU needed."""
import ctypes
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PKG = os.path.join(ROOT, "paper_2607_01308_gb300")

STRUCTS = ("cm_qcache", "cm_qcache_batch", "cm_qcache_query")


def _run(tmp_path, source, *flags):
    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    path, exe = str(tmp_path / "x.c"), str(tmp_path / "x")
    with open(path, "w") as f:
        f.write(source)
    subprocess.run([cc, "-std=c11", "-Wall", "-Wextra", "-Werror", "-pedantic", "-I" + os.path.join(ROOT, "include"), path, *flags, "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr)
    return r.stdout


def test_structs_are_laid_out_as_in_c(tmp_path):
    import paper_2607_01308_gb300 as cm
    fields = [(s, f[0]) for s in STRUCTS for f in getattr(cm, s)._fields_] + [("cm_qcache_query", "reserved")]
    body = "".join('printf("%%s %%zu\\n", "%s", sizeof(%s));\n' % (s, s) for s in STRUCTS)
    body += "".join('printf("%%s.%%s %%zu\\n", "%s", "%s", offsetof(%s, %s));\n' % (s, f, s, f) for s, f in fields)
    out = _run(tmp_path, "#include <stddef.h>\n#include <stdio.h>\n#include \"cm.h\"\nint main(void) {\n%sreturn 0;\n}\n" % body)
    got = dict(line.split() for line in out.splitlines())
    for s in STRUCTS:
        assert int(got[s]) == ctypes.sizeof(getattr(cm, s)), s
    for s, f in fields:
        name = "flags" if (s, f) == ("cm_qcache_query", "reserved") else f
        assert int(got["%s.%s" % (s, f)]) == getattr(getattr(cm, s), name).offset, (s, f)


def test_calls_from_c_refuse_a_missing_context(tmp_path):
    if not os.path.exists(os.path.join(PKG, "libcm.so")):
        pytest.skip("libcm.so not built")
    out = _run(tmp_path, """
#include <stdio.h>
#include <string.h>
#include "cm.h"
#include "cm_testing.h"
int main(void) {
    cm_qcache cache;
    cm_qcache_batch batch;
    /* a descriptor as it was written before it had flags */
    cm_qcache_query query = {.q = NULL, .softmax_scale = 1.0f, .reserved = 0};
    int64_t bytes = 0, counts[2];
    memset(&cache, 0, sizeof cache);
    memset(&batch, 0, sizeof batch);
    if (query.flags != 0 || query.context_lens) return 1;
    if (cm_qcache_schedule(NULL, &batch, NULL, NULL, NULL, 0, NULL, 0, counts, NULL) != CM_ERR_INVALID_ARG) return 2;
    if (cm_qcache_schedule_cut(NULL, &batch, NULL, NULL, NULL, 0, NULL, 0, counts, NULL, NULL) != CM_ERR_INVALID_ARG) return 3;
    if (cm_qcache_append(NULL, &cache, 0, 1, NULL, NULL, 0, 0, 0, NULL, 0, NULL) != CM_ERR_INVALID_ARG) return 4;
    if (cm_qcache_attend(NULL, &cache, 0, &batch, &query, NULL, 0, NULL) != CM_ERR_INVALID_ARG) return 5;
    if (cm_qcache_workspace(NULL, 128, &bytes) != CM_ERR_INVALID_ARG) return 6;
    if (cm_testing_qcache_attend_withheld(NULL, &cache, 0, &batch, &query, NULL, 0, 1, NULL) != CM_ERR_INVALID_ARG) return 7;
    printf("ok %s\\n", cm_last_error_message());
    return 0;
}
""", "-L" + PKG, "-lcm", "-Wl,-rpath," + PKG)
    assert out.startswith("ok") and "context" in out
