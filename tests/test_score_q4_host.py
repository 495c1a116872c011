"""The scores' and the 4-bit layer's calls without a GPU: what they refuse, before any launch, and which launches they make (the
library's host code on a CUDA runtime that runs nothing, tests/helpers/fake_cudart.cu)."""
import ctypes as C

import numpy as np
import pytest

import helpers

OK, INVALID, ALIGNMENT, UNSUPPORTED = 0, -1, -2, -5
F32, BF16 = 0, 1


class Lib:
    def __init__(self):
        self.L, self.kept = helpers.fake_runtime_lib(), []
        self.ctx = C.c_void_p()
        assert self.L.od_create(C.byref(self.ctx), 0, 10, 10, 1, 1) == 0     # (no vocabulary map is needed)
        self.log()

    def close(self):
        assert self.L.od_destroy(self.ctx) == 0

    def buffer(self, nbytes, off=0):
        raw = np.zeros(nbytes + 128, np.uint8)
        self.kept.append(raw)
        return C.c_void_p(raw.ctypes.data + -raw.ctypes.data % 64 + off)

    def log(self):
        return [(w[0].split("_kernel")[0], int(w[1]), int(w[2])) for w in map(str.split, self.L.fake_log().decode().splitlines())]

    def scores(self, B=2, R=3, V=64, dtype=BF16, row=None, seq=None, n_top=2, **p):
        row = V if row is None else row
        a = dict(ctx=self.ctx, logits=self.buffer(64), ids=None, n_rows=None, T=None, logprob=None, entropy=None, row_max=self.buffer(64),
                 row_sum=self.buffer(64), top_ids=self.buffer(64), top_lp=self.buffer(64), flags=None, **{})
        a.update(p)
        return self.L.od_token_logprobs(a["ctx"], B, R, V, a["logits"], dtype, C.c_int64(row), C.c_int64(row * R if seq is None else seq),
                                        a["ids"], a["n_rows"], a["T"], n_top, a["logprob"], a["entropy"], a["row_max"], a["row_sum"],
                                        a["top_ids"], a["top_lp"], a["flags"], None)

    def scores_grad(self, B=2, R=3, V=64, dtype=BF16, row=None, grow=None, n_top=2, **p):
        row = V if row is None else row
        grow = row if grow is None else grow
        a = dict(ctx=self.ctx, logits=self.buffer(64), row_max=self.buffer(64), row_sum=self.buffer(64), entropy=self.buffer(64),
                 top_ids=self.buffer(64), g_lp=None, g_h=None, g_top=None, grad=self.buffer(64))
        a.update(p)
        return self.L.od_token_logprobs_grad(a["ctx"], B, R, V, a["logits"], dtype, C.c_int64(row), C.c_int64(row * R), None, None, None,
                                             a["row_max"], a["row_sum"], a["entropy"], n_top, a["top_ids"], a["g_lp"], a["g_h"], a["g_top"],
                                             a["grad"], C.c_int64(grow), C.c_int64(grow * R), None)

    def q4(self, N=2, V=64, H=128, G=32, dtype=BF16, out_dtype=F32, xs=None, ys=None, backward=False, **p):
        wide, wide_out = (V, H) if backward else (H, V)
        a = dict(ctx=self.ctx, x=self.buffer(64), codes=self.buffer(64), scales=self.buffer(64), out=self.buffer(64))
        a.update(p)
        f = self.L.od_q4_logits_grad if backward else self.L.od_q4_logits
        return f(a["ctx"], N, V, H, G, a["x"], dtype, C.c_int64(wide if xs is None else xs), a["codes"], a["scales"], a["out"], out_dtype,
                 C.c_int64(wide_out if ys is None else ys), None)


@pytest.fixture
def lib():
    x = Lib()
    yield x
    x.close()


def test_scores_refuse(lib):
    odd = lib.buffer(64, 2)
    assert lib.scores() == OK and len(lib.log()) == 1
    for status, kw in [(INVALID, dict(ctx=None)), (INVALID, dict(B=-1)), (INVALID, dict(R=0)), (INVALID, dict(V=0)), (INVALID, dict(n_top=33)),
                       (INVALID, dict(n_top=-1)), (INVALID, dict(top_ids=None)), (INVALID, dict(top_lp=None)), (INVALID, dict(logits=None)),
                       (INVALID, dict(row_max=None)), (INVALID, dict(row_sum=None)), (INVALID, dict(row=56)), (INVALID, dict(seq=64)),
                       (INVALID, dict(B=1 << 20, R=1 << 20)), (INVALID, dict(R=1 << 30, row=1 << 62)), (UNSUPPORTED, dict(dtype=2)),
                       (UNSUPPORTED, dict(V=(1 << 30) + 8)), (ALIGNMENT, dict(logits=odd)), (ALIGNMENT, dict(row=65)), (ALIGNMENT, dict(seq=197))]:
        assert lib.scores(**kw) == status, kw
    assert lib.scores(n_top=0, top_ids=None, top_lp=None) == OK
    lib.log()
    assert lib.scores(B=0, logits=None) == OK and lib.log() == []
    assert not [x for x in lib.log()]


def test_scores_gradient_refuses(lib):
    g, odd = lib.buffer(64), lib.buffer(64, 2)
    assert lib.scores_grad(g_lp=g, g_h=g, g_top=g) == OK and len(lib.log()) == 1
    same = lib.buffer(64)
    assert lib.scores_grad(logits=same, grad=same) == OK
    lib.log()
    for status, kw in [(INVALID, dict(grad=None)), (INVALID, dict(logits=same, grad=same, grow=72)), (INVALID, dict(g_h=g, entropy=None)),
                       (INVALID, dict(g_top=g, top_ids=None)), (INVALID, dict(g_top=g, n_top=0)), (INVALID, dict(n_top=33)),
                       (INVALID, dict(row_sum=None)), (INVALID, dict(grow=56)), (ALIGNMENT, dict(grad=odd)), (ALIGNMENT, dict(grow=65)),
                       (UNSUPPORTED, dict(B=1 << 15, R=1 << 15, V=1 << 20)), (UNSUPPORTED, dict(dtype=2))]:
        assert lib.scores_grad(**kw) == status, kw
    assert lib.log() == []


@pytest.mark.parametrize("backward", [False, True])
def test_q4_refuses(lib, backward):
    odd1, odd2 = lib.buffer(64, 1), lib.buffer(64, 2)
    for status, kw in [(INVALID, dict(ctx=None)), (INVALID, dict(N=-1)), (INVALID, dict(V=0)), (INVALID, dict(H=0)), (INVALID, dict(x=None)),
                       (INVALID, dict(out=None)), (INVALID, dict(codes=None)), (INVALID, dict(scales=None)), (INVALID, dict(H=144)),
                       (INVALID, dict(xs=32)), (INVALID, dict(ys=32)), (UNSUPPORTED, dict(G=16)), (UNSUPPORTED, dict(G=96, H=192)),
                       (UNSUPPORTED, dict(H=65536 + 32)), (UNSUPPORTED, dict(N=65536)), (UNSUPPORTED, dict(dtype=2)), (UNSUPPORTED, dict(out_dtype=7)),
                       (ALIGNMENT, dict(codes=odd2)), (ALIGNMENT, dict(scales=odd1)), (ALIGNMENT, dict(x=odd2)), (ALIGNMENT, dict(out=odd2)),
                       (ALIGNMENT, dict(xs=129)), (ALIGNMENT, dict(ys=129))]:
        assert lib.q4(backward=backward, **kw) == status, kw
    assert lib.log() == []
    assert lib.q4(backward=backward, N=0, x=None, out=None) == OK and lib.log() == []
    assert lib.q4(backward=backward) == OK and len(lib.log()) >= 1


def test_blocks_of_a_row(lib):
    """Eight blocks to a row for one row, one for many; none of a slice below 14 KB."""
    def split(rows, V, dtype=BF16, **kw):
        assert lib.scores(B=rows, R=1, V=V, dtype=dtype, **kw) == OK
        (name, blocks, _), = lib.log()
        assert "od_score" in name and blocks % rows == 0
        return blocks // rows
    assert split(1, 152064) == 8 and split(1, 32000, F32) == 8 and split(1, 32000) == 4 and split(1, 512) == 1
    assert split(96, 128256) == 4 and split(168, 128256) == 2 and split(168, 128256, n_rows=lib.buffer(64)) == 4
    assert split(448, 128256) == 1 and split(1 << 20, 64) == 1


def test_launches_of_the_layer(lib):
    def launches(**kw):
        assert lib.q4(**kw) == OK
        return [(n.split("od_q4")[1].lstrip("_") if "od_q4" in n else n, x, y) for n, x, y in lib.log()]
    # forward: one launch, blocks for the multiprocessors and for tokens
    assert [x[1:] for x in launches(N=1, V=32000, H=768)] == [(148, 1)]
    assert [x[1:] for x in launches(N=1, V=20, H=768)] == [(2, 1)]
    assert [x[1:] for x in launches(N=33, V=32000, H=1024)] == [(148, 2)]
    assert [x[1:] for x in launches(N=33, V=32000, H=4096)] == [(148, 3)]              # 16 tokens fit
    assert [x[1:] for x in launches(N=33, V=32000, H=65536)] == [(148, 5)]             # (none do: 8 at a time)
    # backward: one launch of clusters for a short layer
    (_, blocks, y), = launches(N=8, V=32000, H=768, backward=True)
    assert blocks <= 148 and y == 1
    assert len(launches(N=8, V=16, H=2048, backward=True)) == 1                         # nothing to join
    assert len(launches(N=1, V=304, H=65536, backward=True)) == 1                       # more columns than multiprocessors


@pytest.fixture
def without_clusters():
    """A device with no room for clusters of the gradient's blocks."""
    L = helpers.fake_runtime_lib()
    L.fake_no_driver_functions(1)                           # (what is known of the device is not kept then)
    L.fake_cluster_limit(1)
    yield
    L.fake_cluster_limit(16)
    L.fake_no_driver_functions(0)


def test_the_gradients_join(without_clusters):
    """Where blocks that are no cluster share columns a second kernel joins them, 32 tokens at a time and what is left."""
    lib = Lib()
    assert lib.q4(N=40, V=32000, H=2048, backward=True) == OK
    got = lib.log()
    assert len(got) == 4 and all(b <= 148 and y == 1 for _, b, y in got[0::2])
    assert [x[1:] for x in got[1::2]] == [(2048 // 32, 32), (2048 // 32, 8)]
    lib.close()


def test_kernels_of_the_layer_are_made_ready_when_they_are_first_launched():
    """Not in od_create, which is everybody's; and once to a context."""
    L = helpers.fake_runtime_lib()
    L.fake_limits.restype = C.c_char_p
    L.fake_no_driver_functions(1)                           # (od_create sets the limits of its kernels every time)
    try:
        L.fake_limits()
        lib = Lib()
        created = L.fake_limits().decode().split()
        assert created and not [k for k in created if "od_q4" in k]
        assert lib.scores() == OK and L.fake_limits() == b""
        seen = set()
        for kw in [dict(), dict(H=4096, N=30, V=1000), dict(dtype=F32), dict(G=64), dict(H=65536), dict(backward=True),
                   dict(backward=True, N=40, V=20000, H=2048)]:
            assert lib.q4(**kw) == OK
            ready = set(L.fake_limits().decode().split())
            assert ready and not ready & seen and all("od_q4" in k for k in ready), kw
            assert lib.q4(**kw) == OK and L.fake_limits() == b"", kw
            seen |= ready
        other = Lib()
        assert lib.q4() == OK and not [k for k in L.fake_limits().decode().split() if "od_q4" in k]
        assert other.q4() == OK and [k for k in L.fake_limits().decode().split() if "od_q4" in k]
        other.close()
        lib.close()
    finally:
        L.fake_no_driver_functions(0)


def test_refused_scores_launch_nothing(lib):
    odd = lib.buffer(64, 2)
    for kw in [dict(ctx=None), dict(B=-1), dict(R=0), dict(V=0), dict(n_top=33), dict(n_top=-1), dict(top_ids=None), dict(top_lp=None),
               dict(logits=None), dict(row_max=None), dict(row_sum=None), dict(row=56), dict(seq=64), dict(B=1 << 20, R=1 << 20), dict(dtype=2),
               dict(V=(1 << 30) + 8), dict(logits=odd), dict(row=65), dict(seq=197)]:
        assert lib.scores(**kw) != OK, kw
    assert lib.log() == []
    assert lib.scores(n_top=0, top_ids=None, top_lp=None) == OK and len(lib.log()) == 1
