"""What the library launches for a call, read on a machine without a GPU.

tests/hip_recorder.cpp stands in for the HIP runtime; `run` starts this file
under it with the name of one of the checks below.  Device pointers of the
calls are numbers that nothing reads; the tables that the library uploads are
in host memory and are read here."""
import ctypes
import os
import re
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HERE = os.path.join(ROOT, "tests")


def build(folder):
    """The stand-in, built into `folder`."""
    out = os.path.join(str(folder), "libhiprecorder.so")
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-shared", "-fPIC", "-D__HIP_PLATFORM_AMD__",
                    "-I/opt/rocm/include", os.path.join(HERE, "hip_recorder.cpp"), "-o", out], check=True)
    return out


def run(recorder, check):
    """The check's output; raises with it where the check failed."""
    others = os.environ.get("LD_PRELOAD")  # stay, behind it
    env = dict(os.environ, LD_PRELOAD=recorder + (":" + others if others else ""), HIP_RECORDER=recorder, PYTHONPATH=ROOT)
    p = subprocess.run([sys.executable, os.path.abspath(__file__), check], env=env, cwd=ROOT, text=True,
                       stdout=subprocess.PIPE, stderr=subprocess.STDOUT, timeout=300)
    assert p.returncode == 0, p.stdout[-4000:]
    return p.stdout


# ------------------------------------------------ inside the started process

class Launch:
    def __init__(self, r, i):
        dims = (ctypes.c_uint * 6)()
        r.recorder_dims(i, dims)
        self.r, self.i = r, i
        self.name = r.recorder_name(i).decode()
        self.grid, self.block = list(dims[:3]), list(dims[3:])

    def arg(self, a, kind):
        return ctypes.cast(self.r.recorder_arg(self.i, a), ctypes.POINTER(kind)).contents


class Session:
    def __init__(self):
        self.r = ctypes.CDLL(os.environ["HIP_RECORDER"])
        self.r.recorder_name.restype = ctypes.c_char_p
        self.r.recorder_arg.restype = ctypes.c_void_p
        self.r.recorder_written_after.restype = ctypes.c_longlong
        self.r.recorder_written_after.argtypes = [ctypes.c_void_p]
        self.lib = ctypes.CDLL(os.path.join(ROOT, "paper_2205_14465_amd", "libbytecomp.so"))

    def want(self, part, *kinds):
        sizes = (ctypes.c_size_t * len(kinds))(*[ctypes.sizeof(k) for k in kinds])
        self.r.recorder_want(part.encode(), len(kinds), sizes)

    def take(self):
        """The launches since the last time."""
        out = [Launch(self.r, i) for i in range(self.r.recorder_count())]
        return out

    def clear(self):
        self.r.recorder_clear()


u32, u64, ptr, f32, f64 = ctypes.c_uint32, ctypes.c_uint64, ctypes.c_void_p, ctypes.c_float, ctypes.c_double


def fields(names, kind):
    return [(n, kind) for n in names.split()]


# Layouts of csrc/layers.hpp, as far as they are read here.
class Ortho(ctypes.Structure):
    _fields_ = fields("in_ out momentum", ptr) + fields("ld_in ld_out ld_momentum x xt sym part", u64) + \
        fields("rows cols m n turned parts part0 tile0", u32) + [("step_scale", f32), ("group", u32)]


class OrthoWork(ctypes.Structure):
    _fields_ = fields("matrix tile m n x xt sym part parts sums met", u32)


class OrthoCall(ctypes.Structure):
    _fields_ = [("d", ptr), ("ws", ptr), ("T", ctypes.c_int), ("in_dtype", ctypes.c_int), ("out_dtype", ctypes.c_int),
                ("parts", u32), ("tiles", u32), ("slots", u32), ("meet", u64)]


class StageArgs(ctypes.Structure):
    _fields_ = fields("u v out start", ctypes.c_int) + fields("alpha beta gamma", f32)


GRAM, SYM, NEXT, LAST = range(4)
IDLE = 0xFFFFFFFF


def check_products(s, shapes):
    """Every product launch of the one call since the last clear(): its work list
    lies in what was uploaded, and holds each matrix's tiles once, whole or in all
    their parts, whose slots and counters are nobody else's.  Every matrix of the
    call ends in exactly one last product."""
    last, seen = {}, 0
    for l in s.take():
        if "ortho_product" not in l.name:
            continue
        seen += 1
        side, stage = re.search(r"GemmTileI\w*?Li2ELi(\d+)E.*?ELi(\d)EEEv", l.name).groups()
        side, stage = int(side), int(stage)
        call, at = l.arg(0, OrthoCall), l.arg(2, ptr).value
        count = l.grid[0]
        left = s.r.recorder_written_after(at)
        assert count * ctypes.sizeof(OrthoWork) <= left, f"list of {count} entries, {left} bytes uploaded from its start"
        table = (Ortho * call.T).from_address(call.d)
        assert s.r.recorder_written_after(call.d) >= ctypes.sizeof(table)
        assert sorted((o.rows, o.cols) for o in table) == sorted(x for x in shapes if 0 not in x)
        found, slots, counters = {}, set(), set()
        for w in (OrthoWork * count).from_address(at):
            if w.matrix == IDLE:
                continue
            assert w.matrix < call.T
            o = table[w.matrix]
            assert (w.m, w.n) == (o.m, o.n) and (w.x, w.xt, w.sym) == (o.x >> 8, o.xt >> 8, o.sym >> 8)
            assert w.part < w.parts
            found.setdefault((w.matrix, w.tile), []).append(w)
        for ws in found.values():
            assert sorted(w.part for w in ws) == list(range(ws[0].parts))
            if ws[0].parts > 1:
                assert side == 64 and len({(w.sums, w.met, w.parts) for w in ws}) == 1
                mine = set(range(ws[0].sums, ws[0].sums + ws[0].parts))
                assert not mine & slots and max(mine) < call.slots and ws[0].met not in counters
                assert ws[0].met < call.slots
                slots |= mine
                counters.add(ws[0].met)
        for i in {m for m, _ in found}:
            o = table[i]
            a, b = (o.m + side - 1) // side, (o.n + side - 1) // side
            tiles = a * b if stage in (NEXT, LAST) else a * (a + 1) // 2
            assert sorted(t for m, t in found if m == i) == list(range(tiles))
            if stage == LAST:
                last[i] = last.get(i, 0) + 1
    assert seen and last == {i: 1 for i in range(len([x for x in shapes if 0 not in x]))}, last


def ortho_session():
    from paper_2205_14465_amd import binding as B
    s = Session()
    s.want("ortho_product", OrthoCall, StageArgs, ptr)
    s.lib.bytecomp_orthogonalize.argtypes = [ctypes.c_int, ctypes.POINTER(B.bc_update), ctypes.c_int, ctypes.c_int, ptr,
                                             f64, ptr, ctypes.c_size_t, ptr]
    s.lib.bytecomp_muon_step.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.POINTER(B.bc_param), ctypes.c_int, f64, f64,
                                         ctypes.c_int, f64, ctypes.c_int, ptr, f64, ptr, ctypes.c_size_t, ptr]
    s.abc = (f64 * 3)(*B.MUON_COEFFICIENTS)
    return s, B


def orthogonalize(s, B, dtype, shapes, at=1 << 32, steps=5):
    """The call on matrices at the same places whatever their type."""
    t = (B.bc_update * len(shapes))()
    for i, (r, c) in enumerate(shapes):
        t[i] = B.bc_update(at + (i << 28), at + (1 << 40) + (i << 28), c, c, r, c)
    s.clear()
    rc = s.lib.bytecomp_orthogonalize(dtype, t, len(shapes), steps, s.abc, 1e-7, 1 << 44, 1 << 40, None)
    assert rc == 0, rc


def muon(s, B, wdtype, shapes, at=1 << 32):
    t = (B.bc_param * len(shapes))()
    for i, (r, c) in enumerate(shapes):
        t[i] = B.bc_param(at + (i << 28), at + (1 << 40) + (i << 28), at + (1 << 41) + (i << 28), c, c, c, r, c, 1.0)
    s.clear()
    rc = s.lib.bytecomp_muon_step(wdtype, 0, t, len(shapes), 0.1, 0.9, 1, 0.0, 5, s.abc, 1e-7, 1 << 44, 1 << 40, None)
    assert rc == 0, rc


LISTS = [[(40, 500), (200, 300)], [(32, 32), (64, 64)], [(17, 5000), (150, 150), (63, 640), (640, 64), (5, 0)],
         [(512, 4608)] * 3 + [(2048, 512), (3, 9)], [(31, 63)] * 5, [(768, 768)]]


def work_lists_of_one_type():
    for at, dtype in ((1 << 32, 0), (1 << 33, 1), (1 << 34, 2)):
        s, B = ortho_session()
        for shapes in LISTS:
            orthogonalize(s, B, dtype, shapes, at)
            check_products(s, shapes)


def work_lists_of_the_same_memory_in_another_type():
    s, B = ortho_session()
    for shapes in LISTS:
        for dtype in (0, 1, 0, 2, 1):
            orthogonalize(s, B, dtype, shapes)
            check_products(s, shapes)
    for shapes in LISTS:
        for wdtype in (2, 0, 1, 0):
            muon(s, B, wdtype, shapes)
            check_products(s, shapes)


class LnForward(ctypes.Structure):
    _fields_ = fields("x weight bias y mean rstd", ptr) + fields("rows ldx ldy", u64)


class LnBackward(ctypes.Structure):
    _fields_ = fields("dy x weight mean rstd dx part", ptr) + fields("rows lddy ldx lddx", u64)


def check_rows(launches, rows, bytes_of, kind, names):
    """The launches take the rows one after the other: as many as the grid has
    waves or workgroups for, every pointer at its own row."""
    at = 0
    for l in launches:
        a = l.arg(0, kind)
        threads = 64 if re.search(r"Li64ELi\dE", l.name) else l.block[0]
        assert l.grid[0] * l.block[0] < 1 << 32 and l.grid[1:] == [1, 1]
        assert l.grid[0] * l.block[0] // threads >= a.rows > (l.grid[0] - 1) * l.block[0] // threads
        for n in names:
            assert getattr(a, n) == bytes_of[n][0] + at * bytes_of[n][1], (n, at)
        at += a.rows
    assert at == rows


def layer_norm_rows():
    s = Session()
    s.want("ln_forward", LnForward)
    s.want("ln_backward", LnBackward)
    fwd, bwd = s.lib.bytecomp_layernorm_forward, s.lib.bytecomp_layernorm_backward
    fwd.argtypes = [ctypes.c_int] * 2 + [u64] * 2 + [ptr, u64, ptr, ptr, f64, ptr, u64] + [ptr] * 3
    bwd.argtypes = [ctypes.c_int] * 2 + [u64] * 2 + [ptr, u64, ptr, u64] + [ptr] * 4 + [u64] + [ptr] * 3 + \
        [ctypes.c_size_t, ptr]
    X, Y, Z, M, R, W = (i << 52 for i in range(1, 7))
    for dtype, size in ((0, 4), (1, 2), (2, 2)):
        for cols in (1, 8, 64, 1001, 2048, 2049, 8200, 16384, 70001):
            for rows in (1, 5, (1 << 21) - 1, 1 << 21, (1 << 22) + 1, 1 << 24, (1 << 26) + 5, (1 << 31) - 1):
                s.clear()
                assert fwd(dtype, 0, rows, cols, X, cols + 3, W, W, 1e-5, Y, cols + 5, M, R, None) == 0, (rows, cols)
                places = {"x": (X, (cols + 3) * size), "y": (Y, (cols + 5) * size), "mean": (M, 4), "rstd": (R, 4)}
                check_rows(s.take(), rows, places, LnForward, places)
                s.clear()
                assert bwd(dtype, 0, rows, cols, Z, cols, X, cols + 3, W, M, R, Y, cols + 5, W, W, W, 1 << 50, None) == 0
                wide = [l for l in s.take() if "ln_backward_wide" in l.name]
                assert all(l.grid[0] * l.block[0] < 1 << 32 for l in s.take())
                if wide:
                    places = {"dy": (Z, cols * size), "x": (X, (cols + 3) * size), "dx": (Y, (cols + 5) * size),
                              "mean": (M, 4), "rstd": (R, 4)}
                    check_rows(wide, rows, places, LnBackward, places)
                else:  # the workgroups visit rows a fixed step apart
                    l, = (l for l in s.take() if "ln_backward" in l.name)
                    assert l.arg(0, LnBackward).rows == rows
        # nothing kept
        s.clear()
        assert fwd(dtype, 0, (1 << 26) + 1, 8, X, 8, None, None, 1e-5, Y, 8, None, None, None) == 0
        assert all(l.arg(0, LnForward).mean is None and l.arg(0, LnForward).rstd is None for l in s.take())


if __name__ == "__main__":
    globals()[sys.argv[1]]()
    print("done:", sys.argv[1])
