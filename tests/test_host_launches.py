"""What the vocabulary ends' calls launch, by size (CPU): the built library over a stand-in for the HIP runtime that launches
nothing and writes down what it is asked for (tests/host_launches/recorder.cpp), in a process of its own."""
import json
import os
import shutil
import subprocess
import sys
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# What the scripts below share: they run in another process, in which the stand-in is loaded before the library.
PRELUDE = """
import ctypes as C, json, re, sys, threading
rec = C.CDLL(sys.argv[1], mode=C.RTLD_GLOBAL)
rec.rec_take.restype = rec.rec_kernels.restype = C.c_char_p
rec.rec_finish.argtypes = [C.c_void_p]
import numpy as np
import paper_2602_00482_amd as dta
lib = dta.load_library()
one, none, plenty = C.c_void_p(1 << 20), C.c_void_p(0), 1 << 60     # (addresses that nothing follows)
PER_THREAD = C.c_void_p(2)

def launches():
    '''Launches since the last look: (kernel, kind, rows of the tile's m, of its n, blocks, threads, accepted)'''
    out = []
    for line in rec.rec_take().decode().splitlines():
        if not line.startswith("launch"):
            continue
        _, name, grid, block, ok = line.split()
        kernel = re.search(r"\\d+([a-z_0-9]+?)_kernel", name).group(1)
        kind = next((k for k in ("Bf16", "Parts", "F32") if k in name), "")
        form = re.search(r"FormILi(\\d+)ELi(\\d+)E", name)
        out.append((kernel, kind, *(map(int, form.groups()) if form else (0, 0)), int(grid), int(block), int(ok)))
    return out

def chain(T, vocab, scored=None):
    return dta.tokens_build(dta.tree_build([-1], [T]), np.zeros(T, dtype=np.int32), vocab, scored)

def call(tok, width, dtype, which, stream=none, scale=1.0):
    p = C.byref(dta.VocabParams(width, scale, dtype))
    h = tok.handle
    if which == "embed_fwd": return lib.dta_tree_embed_fwd(h, p, one, one, stream)
    if which == "embed_bwd": return lib.dta_tree_embed_bwd(h, p, one, one, 0, one, plenty, stream)
    if which == "logprob_fwd": return lib.dta_tree_logprob_fwd(h, p, one, one, one, one, one, plenty, stream)
    return lib.dta_tree_logprob_bwd(h, p, one, one, one, one, one, one, 0, one, plenty, stream)
"""


@pytest.fixture(scope="module")
def recorded():
    """recorded(script, *args): what the script prints as JSON, with the stand-in loaded."""
    gxx = shutil.which("g++")
    include = "/opt/rocm/include"
    if gxx is None or not os.path.exists(os.path.join(include, "hip", "hip_runtime_api.h")):
        pytest.skip("no g++ or no HIP headers")
    work = tempfile.mkdtemp(prefix="dta_launches_")
    out = os.path.join(work, "recorder.so")
    res = subprocess.run([gxx, "-std=c++17", "-O1", "-shared", "-fPIC", "-I", include,
                          os.path.join(ROOT, "tests", "host_launches", "recorder.cpp"), "-o", out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr

    def run(script, *args):
        res = subprocess.run([sys.executable, "-c", PRELUDE + script, out, *map(str, args)], capture_output=True, text=True,
                             timeout=300, cwd=ROOT)
        assert res.returncode == 0, res.stderr[-4000:]
        return json.loads(res.stdout.splitlines()[-1])

    yield run
    shutil.rmtree(work, ignore_errors=True)


# rows x ids of 2^37 to 2^40: more threads than a launch may have in one launch of the logits
MANY = [(2 ** 21, 2 ** 18, 64, "bf16"), (2 ** 22, 131072, 1024, "bf16"), (2 ** 20, 2 ** 18, 64, "f32"),
        (2 ** 21, 2 ** 18 + 77, 192, "f32"), (2 ** 23 + 5, 100003, 64, "bf16"), (1000, 2 ** 24 - 1, 64, "bf16")]


@pytest.mark.parametrize("rows,vocab,width,dtype", MANY)
def test_no_launch_of_a_large_call_is_too_large(recorded, rows, vocab, width, dtype):
    """Every launch has fewer than 2^32 threads, and the launches of the logits cover all rows and ids."""
    got = recorded("""
rows, vocab, width, dtype = int(sys.argv[2]), int(sys.argv[3]), int(sys.argv[4]), dict(f32=dta.F32, bf16=dta.BF16)[sys.argv[5]]
tok = chain(rows + 1, vocab)
out = {}
for which in ("logprob_fwd", "logprob_bwd", "embed_fwd", "embed_bwd"):
    status = call(tok, width, dtype, which)
    out[which] = (status, launches())
print(json.dumps(out))
""", rows, vocab, width, dtype)
    for which, (status, all_) in got.items():
        assert status == 0, which
        assert all(grid * block < 2 ** 32 and ok for _, _, _, _, grid, block, ok in all_), (which, all_)
    for kind in ("Bf16",) if dtype == "bf16" else {k[1] for k in got["logprob_fwd"][1] if k[0] == "logits_fwd"}:
        tiles = sum(g * m * n for kernel, kd, m, n, g, _, _ in got["logprob_fwd"][1] if kernel == "logits_fwd" and kd == kind)
        assert rows * vocab <= tiles <= (rows + 256) * (vocab + 256 * 64), kind


@pytest.mark.parametrize("tokens", [2 ** 24 - 1, 2 ** 24 - 62, 2 ** 24 - 63])
def test_rows_up_to_the_largest_number(recorded, tokens):
    """Rows of the tree are gathered by a block of 256 threads each, padded to 64 rows: 2^32 threads in one launch."""
    got = recorded("""
T = int(sys.argv[2])
tok = chain(T, 100)
out = []
for dtype in (dta.F32, dta.BF16):
    for which, k in (("logprob_fwd", dta.VOCAB_LOGPROB_FWD), ("logprob_bwd", dta.VOCAB_LOGPROB_BWD)):
        out.append((call(tok, 64, dtype, which), dta.vocab_workspace_bytes(tok, dta.VocabParams(64, 1.0, dtype), k), launches()))
print(json.dumps(out))
""", tokens)
    for status, workspace, all_ in got:
        assert status == 0 and workspace > 0 and all_
        assert all(grid * block < 2 ** 32 and ok for _, _, _, _, grid, block, ok in all_), all_


@pytest.mark.parametrize("dtype,width,tokens", [("f32", 1088, 2 ** 33 // 1088), ("f32", 64, 2 ** 27 - 1), ("bf16", 1088, 2 ** 33 // 1088)])
def test_embeddings_of_the_largest_tensors(recorded, dtype, width, tokens):
    """Tensors of just under 2^33 elements whose rows fill a block's threads worst, or best, and ids that all occur but one."""
    got = recorded("""
T, width, dtype = int(sys.argv[2]), int(sys.argv[3]), dict(f32=dta.F32, bf16=dta.BF16)[sys.argv[4]]
ids = np.arange(T, dtype=np.int32)
ids[-1] = 0
tok = dta.tokens_build(dta.tree_build([-1], [T]), ids, T)
print(json.dumps([(call(tok, width, dtype, which), launches()) for which in ("embed_fwd", "embed_bwd")]))
""", tokens if width > 64 else tokens // 8, width, dtype)   # (rows of 64: an eighth, for the host's memory)
    for status, all_ in got:
        assert status == 0 and len(all_) == 1 and all_[0][4] * all_[0][5] < 2 ** 32, all_


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_call_ends_at_a_launch_that_fails(recorded, dtype):
    """Nothing is launched behind a launch that the runtime refuses, the call says so, and the tables' memory is not given to
    another upload before the launches in front of it have run."""
    got = recorded("""
dtype = dict(f32=dta.F32, bf16=dta.BF16)[sys.argv[2]]
S = C.c_void_p(0x1000)
ids = np.zeros(3001, dtype=np.int32)                      # (one id many times: sums in parts, two launches)
build = lambda: dta.tokens_build(dta.tree_build([-1], [3001]), ids, 20000)
def upload(tok):
    tok.prepare()
    return [int(l.split()[1]) for l in rec.rec_take().decode().splitlines() if l.startswith("copy")][0]
out = []
for which in ("embed_fwd", "embed_bwd", "logprob_fwd", "logprob_bwd"):
    tok = build()
    tok.prepare()
    rec.rec_take()
    assert call(tok, 512, dtype, which, S) == 0
    n = len(launches())
    rec.rec_finish(S)
    tok.destroy()
    for k in range(1, n + 1):
        rec.rec_finish(S)
        tok = build()
        block = upload(tok)
        rec.rec_fail(k)
        status = call(tok, 512, dtype, which, S)
        tried = launches()
        tok.destroy()
        others, after = [build() for _ in range(40)], build()
        while_running = block in [upload(o) for o in others]     # (all that is free is taken)
        rec.rec_finish(S)
        then = while_running or upload(after) == block
        for o in others + [after]:
            o.destroy()
        out.append((which, n, k, status, [t[-1] for t in tried], while_running, then))
print(json.dumps(out))
""", dtype)
    assert {(w, n) for w, n, *_ in got} >= {("embed_fwd", 1), ("embed_bwd", 2)}
    for which, n, k, status, tried, while_running, then in got:
        assert status == -5 and tried == [1] * (k - 1) + [0], (which, n, k, status, tried)
        # (a call whose first launch fails has left nothing that reads the tables)
        assert then and while_running == (k == 1), (which, n, k)


@pytest.mark.parametrize("stream", [0, 2, 0x1000])
def test_calls_of_two_threads_on_streams_of_one_handle(recorded, stream):
    """hipStreamPerThread (2) is one handle and a stream of its own in every thread: the tables' memory is given to another
    upload when the calls of both threads have run.  On a stream that the threads share the later call says it for both."""
    got = recorded("""
S = C.c_void_p(int(sys.argv[2]))
build = lambda: chain(3000, 20000)
def upload(tok):
    tok.prepare()
    return [int(l.split()[1]) for l in rec.rec_take().decode().splitlines() if l.startswith("copy")][0]
tok = build()
block = upload(tok)
called, over, step = threading.Event(), threading.Event(), []
def first():
    step.append(call(tok, 64, dta.BF16, "embed_fwd", S))
    called.set()
    over.wait()
    rec.rec_finish(S)
def second():
    step.append(call(tok, 64, dta.BF16, "embed_fwd", S))
    rec.rec_finish(S)
a = threading.Thread(target=first)
a.start()
called.wait()
b = threading.Thread(target=second)
b.start()
b.join()
tok.destroy()
rec.rec_take()
other, third = build(), build()
one_ran = upload(other) == block
over.set()
a.join()
both_ran = one_ran or upload(third) == block
print(json.dumps([step, one_ran, both_ran]))
""", stream)
    assert got == [[0, 0], stream != 2, True]


@pytest.mark.parametrize("dtype,size", [("bf16", 2), ("f32", 4)])
def test_which_embeddings_are_stored_past_the_cache(recorded, dtype, size):
    """Both sides of the measured crossings: results of 240 and 270 MiB of embeddings, 360 and 410 MiB of a table's gradient,
    whatever the other tensor has; an accumulator is added to by plain stores."""
    got = recorded("""
dtype, size = dict(f32=dta.F32, bf16=dta.BF16)[sys.argv[2]], int(sys.argv[3])
out = []
def stream(which, T, vocab):
    tok = chain(T, vocab)
    assert call(tok, 1024, dtype, which) == 0
    name = [l.split()[1] for l in rec.rec_take().decode().splitlines() if l.startswith("launch")][0]
    return "Lb1" in name
rows = lambda mib: mib * 1024 // size
for other in (10, 10000, 300000):
    out.append([stream("embed_fwd", rows(m), other) for m in (100, 240, 270, 900)])
    out.append([stream("embed_bwd", other, rows(m)) for m in (200, 360, 410, 900)])
print(json.dumps(out))
""", dtype, size)
    assert got == [[False, False, True, True]] * 6


def test_the_gpu_tests_reach_every_kernel_of_the_log_probabilities(recorded):
    """The sizes of tests/test_gpu_vocab_forms.py take every kernel of dta_logprob.hip that the library has: no instance is
    without a test, and none without a call."""
    import test_gpu_vocab_forms as G
    missing, every = recorded("""
rec.rec_take()
every = {n for n in rec.rec_kernels().decode().split() if re.search(r"(logits_fwd|logits_bwd|lse|gather|split|clear|grad|outer|sum)_kernel", n)}
every = {n for n in every if "dta_f32" not in n and "attn" not in n}
left = set(every)
for dtype, rows, vocab, width in json.loads(sys.argv[2]):
    tok = chain(rows + 1, vocab)
    for which in ("logprob_fwd", "logprob_bwd"):
        assert call(tok, width, dict(f32=dta.F32, bf16=dta.BF16)[dtype], which) == 0
    left -= {l.split()[1] for l in rec.rec_take().decode().splitlines() if l.startswith("launch")}
print(json.dumps([sorted(left), sorted(every)]))
""", json.dumps(G.FORMS))
    assert len(every) > 50 and missing == []


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_workspaces_hold_what_the_header_says(recorded, dtype):
    """The terms of the header on calls that are split, or not, into parts, and into blocks of the vocabulary."""
    size = 4 if dtype == "f32" else 2
    shapes = [(rows, vocab, width) for rows in (1, 100, 129, 3000, 50000, 1 << 20) for vocab in (500, 32000, 200003)
              for width in (64, 1024, 4096)] + [(40000, 1000, 32768), (1 << 21, 3000, 4000 // 64 * 64)]
    got = recorded("""
dtype = dict(f32=dta.F32, bf16=dta.BF16)[sys.argv[2]]
out = []
toks = {}
for rows, vocab, width in json.loads(sys.argv[3]):
    if (rows, vocab) not in toks:
        toks.clear()
        toks[rows, vocab] = chain(rows + 1, vocab)
    p = dta.VocabParams(width, 1.0, dtype)
    out.append([dta.vocab_workspace_bytes(toks[rows, vocab], p, k) for k in (2, 3)])
print(json.dumps(out))
""", dtype, json.dumps(shapes))
    up = lambda x, to: -(-x // to) * to
    for (rows, vocab, width), (fwd, bwd) in zip(shapes, got):
        R, T, GiB2 = up(rows, 64), rows + 1, 1 << 31
        ids = min(up(vocab, 256), max(256, GiB2 // (6 * width)))
        pairs, slack = 8 * rows * -(-vocab // 128), 8192
        copied = R * width * size if T * width * size >= 1 << 32 else 0
        plain, parts = pairs + copied + slack, pairs + copied + 6 * R * width + 6 * width * ids + slack
        assert fwd <= (parts if dtype == "f32" else plain), (rows, vocab, width, fwd)
        few = dtype == "bf16" and rows <= 128
        R = up(rows, 256)
        least = rows * width * size * (2 if few else 1) + 4 * rows * width          # the rows, one sum of d_hidden
        dz = lambda b: R * b * min(up(vocab, 256), max(256, GiB2 // (R * b)))
        each = (4 if few else 2) if dtype == "bf16" else 6
        most = R * width * size * (2 if few else 1) + max(dz(each), dz(4)) + 64 * 4 * width * (R + min(up(vocab, 256), max(256, GiB2 // (2 * R)))) + \
            (6 * R * width + 6 * width * ids if dtype == "f32" else 0) + 8 * R + slack
        assert least <= bwd <= most, (rows, vocab, width, bwd, least, most)
