"""Device memory, streams and graphs for the tests of operators on device data: plain calls of the HIP runtime that the library links."""
import ctypes as C

import numpy as np

from paper_2504_19516_amd import synth

NP = {"f32": np.float32, "bf16": np.uint16, "f16": np.float16, "i32": np.int32}


def rounded(x, dtype):
    """x (any float array) in the precision of `dtype`, as float32."""
    x = np.asarray(x, np.float32)
    if dtype == "bf16":
        b = x.view(np.uint32)
        r = ((b + 0x7FFF + ((b >> 16) & 1)) & 0xFFFF0000).astype(np.uint32).view(np.float32)
        return np.where(np.isnan(x), np.float32(np.nan), r).astype(np.float32)
    return x.astype(np.float16).astype(np.float32) if dtype == "f16" else x


def stored(x, dtype):
    """The bits of a float array (already in that precision) in memory."""
    return (np.asarray(x, np.float32).view(np.uint32) >> 16).astype(np.uint16) if dtype == "bf16" else np.asarray(x, np.float32).astype(NP[dtype])


def widened(raw, dtype):
    return (raw.astype(np.uint32) << 16).view(np.float32) if dtype == "bf16" else raw.astype(np.float32)


class Device:
    """Everything allocated is freed by close()."""

    def __init__(self):
        from paper_2504_19516_amd import sts
        sts.lib()
        self.rt = C.CDLL("libamdhip64.so")
        self.bufs, self.streams = [], []

    def __enter__(self):
        return self

    def __exit__(self, *a):
        self.sync()
        for p in self.bufs:
            self.rt.hipFree(C.c_void_p(p))
        for s in self.streams:
            self.rt.hipStreamDestroy(C.c_void_p(s))

    def ck(self, rc, what):
        assert rc == 0, f"{what}: hip error {rc}"

    def alloc(self, nbytes):
        p = C.c_void_p()
        self.ck(self.rt.hipMalloc(C.byref(p), C.c_size_t(max(int(nbytes), 1))), "hipMalloc")
        self.bufs.append(p.value)
        return p.value

    def write(self, p, arr):
        arr = np.ascontiguousarray(arr)
        if arr.nbytes:
            self.ck(self.rt.hipMemcpy(C.c_void_p(p), arr.ctypes.data_as(C.c_void_p), C.c_size_t(arr.nbytes), 1), "hipMemcpy")

    def put(self, arr, dtype=None, offset=0):
        """A device copy, `offset` bytes behind an address that is aligned to 256; dtype "bf16" or "f16": of floats in that precision."""
        arr = stored(arr, dtype) if dtype in ("bf16", "f16") else np.ascontiguousarray(arr)
        p = self.alloc(arr.nbytes + offset) + offset
        self.write(p, arr)
        return p

    def ints(self, values):
        return self.put(np.asarray(values, np.int32))

    def get(self, p, shape, dtype):
        """dtype: of NP, "bf16" and "f16" come back widened."""
        out = np.empty(shape, NP[dtype])
        if out.nbytes:
            self.ck(self.rt.hipMemcpy(out.ctypes.data_as(C.c_void_p), C.c_void_p(p), C.c_size_t(out.nbytes), 2), "hipMemcpy")
        return widened(out, dtype) if dtype in ("bf16", "f16") else out

    def sync(self):
        self.ck(self.rt.hipDeviceSynchronize(), "hipDeviceSynchronize")

    def stream(self):
        s = C.c_void_p()
        self.ck(self.rt.hipStreamCreateWithFlags(C.byref(s), 1), "hipStreamCreate")       # does not wait for the null stream
        self.streams.append(s.value)
        return s.value

    def graph(self, stream, calls):
        """calls() captured on the stream; returns a function that launches it there."""
        g, x = C.c_void_p(), C.c_void_p()
        self.ck(self.rt.hipStreamBeginCapture(C.c_void_p(stream), 2), "hipStreamBeginCapture")
        calls()
        self.ck(self.rt.hipStreamEndCapture(C.c_void_p(stream), C.byref(g)), "hipStreamEndCapture")
        self.ck(self.rt.hipGraphInstantiate(C.byref(x), g, None, None, C.c_size_t(0)), "hipGraphInstantiate")
        return lambda: self.ck(self.rt.hipGraphLaunch(x, C.c_void_p(stream)), "hipGraphLaunch")


def pool_of(k, v, tables, lens, pages, dtype, behind=0.0, rng=None):
    """One layer's pool [pages][n_kv][K: 16 x d | V^T: d x 16] as floats: k, v lists of [len, n_kv, d] by request. Whatever no token fills holds
    `behind` (a value, or "noise")."""
    n_kv, d = k[0].shape[1:]
    pool = np.full((pages, n_kv, 2 * 16 * d), behind, np.float32) if behind != "noise" else rng.standard_normal((pages, n_kv, 2 * 16 * d)).astype(np.float32)
    kp, vp = pool[:, :, :16 * d].reshape(pages, n_kv, 16, d), pool[:, :, 16 * d:].reshape(pages, n_kv, d, 16)
    for r, n in enumerate(lens):
        for t in range(n):
            p = tables[r][t // 16]
            kp[p, :, t % 16] = k[r][t]
            vp[p, :, :, t % 16] = v[r][t]
    out = np.concatenate([kp.reshape(pages, n_kv, -1), vp.reshape(pages, n_kv, -1)], axis=2)
    return rounded(out, dtype)


__all__ = ["Device", "NP", "pool_of", "rounded", "stored", "widened", "synth"]
