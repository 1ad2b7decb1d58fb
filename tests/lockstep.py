"""The kernels of draws, largest logits, gradient norm and clipping on the CPU (tests/lanes): built from their own sources and called through the C ABI on host memory. A workgroup's wavefronts run one
after the other, in an order of choice, each as far as it gets without the others: what a wait is missing for goes wrong every time."""
import ctypes as C
import os
import subprocess

import numpy as np

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CXX = "/opt/rocm/llvm/bin/clang++"
ORDERS = (0, 1, 2)      # the first wavefront first, the last one, at random


def build(to):
    """The library, built into the folder `to` (about ten seconds)."""
    lanes, csrc = os.path.join(ROOT, "tests", "lanes"), os.path.join(ROOT, "paper_2504_07878_amd", "csrc")
    sources = [os.path.join(lanes, "lanes.cpp")] + [os.path.join(csrc, f"{x}.hip") for x in ("row_pick_api", "row_pick_kernels", "clip_api", "clip_kernels")]
    objects = [os.path.join(to, os.path.basename(s) + ".o") for s in sources]
    flags = ["-x", "c++", "-std=c++17", "-O1", "-ffp-contract=off", "-fPIC", "-I", lanes]
    for p in [subprocess.Popen([CXX, *flags, "-c", s, "-o", o]) for s, o in zip(sources, objects)]:
        assert p.wait() == 0
    path = os.path.join(to, "liblanes.so")
    subprocess.run([CXX, "-shared", "-o", path, *objects], check=True)
    return Library(path)


def room(nbytes):
    """Memory on a multiple of 256 bytes, with something in it."""
    buf = np.full(nbytes + 256, 0xa5, np.uint8)
    at = -buf.ctypes.data % 256
    return buf[at:at + nbytes]


class Library:
    def __init__(self, path):
        from paper_2504_07878_amd import tokroute as tr
        self.tr, self.lib = tr, C.CDLL(path)
        for f in (self.lib.tr_pick_workspace_bytes, self.lib.tr_grad_workspace_bytes):
            f.restype = C.c_size_t
        self.lib.lanes_order.argtypes = [C.c_uint64]
        self.lib.lanes_message.restype, self.lib.lanes_launches.restype, self.lib.lanes_launches.argtypes = C.c_char_p, C.c_long, [C.c_char_p]

    def _done(self, rc):
        assert rc == 0, (rc, self.lib.lanes_message())

    def _rows(self, z, order):
        """z: float32 [n][v], or the bit patterns of bfloat16 (uint16)."""
        tr, (n, v) = self.tr, z.shape
        cfg = tr.tr_pick_config(n, v, tr.BF16 if z.dtype == np.uint16 else tr.F32)
        rows = tr.tr_pick_rows(z.ctypes.data, z.strides[0] // z.itemsize, n)
        ws = room(self.lib.tr_pick_workspace_bytes(C.byref(cfg)))
        self.lib.lanes_order(order)
        self.lib.lanes_launches(None)
        return cfg, rows, ws

    def sample(self, z, u, order=0, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
        cfg, rows, ws = self._rows(z, order)
        u = np.ascontiguousarray(u, dtype=np.float32)
        token, logprob = np.full(len(z), 77, np.int32), np.full(len(z), 77, np.float32)
        how = self.tr.tr_sample_how(u.ctypes.data, None, None, None, None, temperature, top_k, top_p, min_p)
        self._done(self.lib.tr_sample(C.byref(cfg), C.c_void_p(ws.ctypes.data), C.c_size_t(ws.nbytes), None, C.byref(rows), C.byref(how), C.c_void_p(token.ctypes.data), C.c_void_p(logprob.ctypes.data)))
        return token, logprob

    def top(self, z, k, order=0):
        cfg, rows, ws = self._rows(z, order)
        ids, values = np.full((len(z), k), 77, np.int32), np.full((len(z), k), 77, np.float32)
        self._done(self.lib.tr_top(C.byref(cfg), C.c_void_p(ws.ctypes.data), C.c_size_t(ws.nbytes), None, C.byref(rows), k, C.c_void_p(ids.ctypes.data), C.c_void_p(values.ctypes.data)))
        return ids, values

    def launches(self, part):
        """Launches of kernels of that name in the last call."""
        return self.lib.lanes_launches(part.encode())

    def clip(self, grads, max_norm, out=None, order=0):
        """grads: flat arrays, float32 or the bit patterns of bfloat16 (uint16); out: the same. None: in place; max_norm None: the norm alone."""
        n, tr = len(grads), self.tr
        at = lambda arrays: (C.c_void_p * n)(*[x.ctypes.data for x in arrays])   # noqa: E731
        counts, types = (C.c_int64 * n)(*[x.size for x in grads]), (C.c_int32 * n)(*[tr.BF16 if x.dtype == np.uint16 else tr.F32 for x in grads])
        ws, norm = room(self.lib.tr_grad_workspace_bytes()), np.full(1, 77, np.float32)
        ends = C.c_void_p(ws.ctypes.data), C.c_size_t(ws.nbytes), None, n, at(grads)
        self.lib.lanes_order(order)
        self.lib.lanes_launches(None)
        if max_norm is None:
            self._done(self.lib.tr_grad_norm(*ends, counts, types, C.c_void_p(norm.ctypes.data)))
        else:
            self._done(self.lib.tr_grad_clip(*ends, at(grads if out is None else out), counts, types, C.c_float(max_norm), C.c_void_p(norm.ctypes.data)))
        return norm[0]
