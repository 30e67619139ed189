"""Thin ctypes binding of libmorello_mi355x.so (include/morello_mi355x.h).

Argument marshalling only: every step of the hot path runs in the library's
HIP kernels.  PyTorch supplies device memory and the stream.  There is no CPU
fallback: importing works without a GPU, calling `solve` does not.
"""
import ctypes as C
import os
import struct

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libmorello_mi355x.so")

INF = (1 << 64) - 1
NONE = 0xFFFF
MAX_DIMS = 16
NOALLOC_MAX_QUERIES = 4096

OK, E_INVAL, E_NOMEM, E_HIP, E_RANGE, E_BUFSZ, E_OVERFLOW = 0, -1, -2, -3, -4, -5, -6

EXPORTS = ["mrl_target_create", "mrl_target_destroy", "mrl_geometry", "mrl_table_bytes", "mrl_solve", "mrl_solve_graph",
           "mrl_table_destroy", "mrl_query", "mrl_query_noalloc", "mrl_query_compressed", "mrl_rewrite_decode", "mrl_coord_of_spec",
           "mrl_emit_compressed", "mrl_schedule", "mrl_copy_dense", "mrl_linear_bytes", "mrl_linear", "mrl_linear_grad_bytes",
           "mrl_linear_grad", "mrl_dropout", "mrl_layer_norm", "mrl_layer_norm_grad_bytes", "mrl_layer_norm_grad", "mrl_mx_quantize",
           "mrl_mx_dequantize", "mrl_mx_linear_bytes", "mrl_mx_linear", "mrl_spec_linear", "mrl_last_error"]


class MorelloError(RuntimeError):
    def __init__(self, code, msg):
        super().__init__("mrl error %d: %s" % (code, msg))
        self.code = code


class _Microkernel(C.Structure):
    _fields_ = [("kind", C.c_uint32), ("lanes", C.c_uint32), ("cost", C.c_uint64)]


class _TargetDesc(C.Structure):
    _fields_ = [("n_levels", C.c_uint32),
                ("capacity_bytes", C.c_uint64 * 4),
                ("load_coef", C.c_uint32 * 2 * 4 * 4),
                ("store_coef", C.c_uint32 * 2 * 4 * 4),
                ("convert_coef", C.c_uint32),
                ("zero_coef", C.c_uint32 * 4),
                ("loop_overhead", C.c_uint32),
                ("n_microkernels", C.c_uint32),
                ("mk", _Microkernel * 8),
                ("threads", C.c_uint32),
                ("sync_cost", C.c_uint32),
                ("level_weight", C.c_uint32 * 4),
                ("line_bytes", C.c_uint32),
                ("strip", C.c_uint32)]


class _LatticeDesc(C.Structure):
    _fields_ = [("kind", C.c_uint32),
                ("n_sizes", C.c_uint32 * 4),
                ("sizes", C.POINTER(C.c_uint32) * 4),
                ("layout_coord", C.c_uint8 * 5),
                ("dtype_coord", C.c_uint8 * 5),
                ("base_dtype_bytes", C.c_uint8 * 5)]


class Stats(C.Structure):
    _fields_ = [("n_specs", C.c_uint64), ("n_admissible", C.c_uint64), ("n_rewrites", C.c_uint64),
                ("n_levels_run", C.c_uint32), ("fill_ms", C.c_float), ("compress_ms", C.c_float),
                ("n_decision_boxes", C.c_uint64), ("n_cost_boxes", C.c_uint64),
                ("scratch_used", C.c_uint64), ("prefill_ms", C.c_float)]

    def as_dict(self):
        return {k: getattr(self, k) for k, _ in self._fields_}


class _Coord(C.Structure):
    _fields_ = [("x", C.c_uint32 * MAX_DIMS)]


class _ScheduleNode(C.Structure):
    _fields_ = [("table", C.c_uint32), ("rewrite", C.c_uint16), ("n_children", C.c_uint16),
                ("cost", C.c_uint64), ("spec", _Coord)]


class Rewrite(C.Structure):
    _fields_ = [("cls", C.c_uint8), ("operand_or_dim", C.c_uint8), ("dst_level", C.c_uint8),
                ("transposed", C.c_uint8), ("convert", C.c_uint8),
                ("tile_size", C.c_uint32), ("mk_index", C.c_uint32)]


BOX_DTYPE = np.dtype([("lo", np.uint16, (MAX_DIMS,)), ("hi", np.uint16, (MAX_DIMS,)),
                      ("v0", np.uint64), ("v1", np.uint64)])

_lib = None


def lib():
    """Load the built library; raises if it has not been built (no fallback)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise ImportError("%s is missing: run __graft_entry__.build() (hipcc, gfx950)" % LIB_PATH)
        # torch first: it brings its own HIP runtime, and the library must share that one.  Loaded the
        # other way round the process holds two runtimes and the library's finds no device.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        _lib = C.CDLL(LIB_PATH)
        for name in EXPORTS:
            getattr(_lib, name).restype = C.c_int32
        _lib.mrl_last_error.restype = C.c_char_p
        _lib.mrl_target_destroy.restype = None
        _lib.mrl_table_destroy.restype = None
        # (the operators' calls are short: with these, plain integers and bytes go in without an object each)
        for name in ("mrl_linear", "mrl_linear_grad", "mrl_layer_norm_grad", "mrl_mx_linear"):
            getattr(_lib, name).argtypes = [C.c_char_p, C.c_void_p, C.c_size_t, C.c_void_p]
            getattr(_lib, name + "_bytes").argtypes = [C.c_char_p, C.c_void_p]
        for name in ("mrl_dropout", "mrl_layer_norm", "mrl_mx_quantize", "mrl_mx_dequantize"):
            getattr(_lib, name).argtypes = [C.c_char_p, C.c_void_p]
    return _lib


def _check(rc):
    if rc != 0:
        raise MorelloError(rc, lib().mrl_last_error().decode())


def _target_desc(t):
    d = _TargetDesc()
    d.n_levels = t["n_levels"]
    for l in range(4):
        d.capacity_bytes[l] = t["capacity_bytes"][l]
        d.zero_coef[l] = t["zero_coef"][l]
        for k in range(4):
            for x in range(2):
                d.load_coef[l][k][x] = t["load_coef"][l][k][x]
                d.store_coef[l][k][x] = t["store_coef"][l][k][x]
    d.convert_coef = t["convert_coef"]
    d.loop_overhead = t["loop_overhead"]
    d.n_microkernels = len(t["microkernels"])
    for j, (kind, lanes, cost) in enumerate(t["microkernels"][:8]):
        d.mk[j].kind, d.mk[j].lanes, d.mk[j].cost = kind, lanes, cost
    d.threads = t.get("threads", 1)
    d.sync_cost = t.get("sync_cost", 0)
    for l in range(4):
        d.level_weight[l] = t.get("level_weight", [0, 0, 0, 0])[l]
    d.line_bytes = t.get("line_bytes", 0)
    d.strip = t.get("strip", 0)
    return d


def _lattice_desc(lat):
    d = _LatticeDesc()
    d.kind = lat["kind"]
    keep = []
    for a in range(4):
        arr = (C.c_uint32 * max(1, len(lat["sizes"][a])))(*lat["sizes"][a])
        keep.append(arr)
        d.n_sizes[a] = len(lat["sizes"][a])
        d.sizes[a] = C.cast(arr, C.POINTER(C.c_uint32))
    for i in range(5):
        d.layout_coord[i] = lat["layout_coord"][i]
        d.dtype_coord[i] = lat["dtype_coord"][i]
        d.base_dtype_bytes[i] = lat["base_dtype_bytes"][i]
    d._keep = keep
    return d


class Target:
    def __init__(self, desc):
        self._h = C.c_void_p()
        _check(lib().mrl_target_create(C.byref(_target_desc(desc)), C.byref(self._h)))

    def close(self):
        if self._h:
            lib().mrl_target_destroy(self._h)
            self._h = C.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def geometry(target, lattice, desc=None):
    """(extents, number of Specs); desc: the lattice's descriptor if the caller has built it."""
    nd, n = C.c_uint32(), C.c_uint64()
    ext = (C.c_uint32 * MAX_DIMS)()
    L = _lattice_desc(lattice) if desc is None else desc
    _check(lib().mrl_geometry(target._h, C.byref(L), C.byref(nd), ext, C.byref(n)))
    return list(ext[:nd.value]), n.value


def table_bytes(target, lattice):
    a, b, c = C.c_size_t(), C.c_size_t(), C.c_size_t()
    _check(lib().mrl_table_bytes(target._h, C.byref(_lattice_desc(lattice)), C.byref(a), C.byref(b), C.byref(c)))
    return a.value, b.value, c.value


class Table:
    """A solved table.  Holds the torch tensors that back it."""

    def __init__(self, handle, target, lattice, extents, tensors, stats, deps=()):
        self._h, self.target, self.lattice = handle, target, lattice
        self.extents, self._tensors, self.stats = extents, tensors, stats
        self._deps = tuple(deps)        # keeps the tables this one was solved against alive
        self.n_specs = int(np.prod(extents, dtype=np.uint64))

    def close(self):
        if self._h:
            lib().mrl_table_destroy(self._h)
            self._h = C.c_void_p()
            self._tensors = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def query(self, coords, compressed=False, noalloc=False):
        """(cost, rewrite id) of the Specs at `coords`; compressed=True answers from the two box
        lists alone (mrl_query_compressed) instead of the dense table; noalloc=True asks through
        mrl_query_noalloc (at most NOALLOC_MAX_QUERIES coordinates)."""
        if not (isinstance(coords, np.ndarray) and coords.dtype.kind in "iu"):
            coords = np.asarray(coords, dtype=np.uint32)
        coords = coords.reshape(-1, len(self.extents))
        n = len(coords)
        buf = np.zeros((n, MAX_DIMS), dtype=np.uint32)
        buf[:, :coords.shape[1]] = coords             # (integers of other widths are converted in this one pass)
        cost = np.empty(n, dtype=np.uint64)
        rw = np.empty(n, dtype=np.uint16)
        fn = lib().mrl_query_compressed if compressed else lib().mrl_query_noalloc if noalloc else lib().mrl_query
        _check(fn(self._h, buf.ctypes.data_as(C.POINTER(_Coord)), C.c_size_t(n),
                  cost.ctypes.data_as(C.POINTER(C.c_uint64)), rw.ctypes.data_as(C.POINTER(C.c_uint16))))
        return cost, rw

    def schedule(self, coord):
        """Program of the Spec at `coord`: [(table, coord, rewrite id, cost, children)] in
        pre-order; table 0 = this table, 1 + i = the i-th table it was solved against, 3 + i = the
        i-th table that one's second dep was solved against."""
        goal = _Coord()
        for a, v in enumerate(coord):
            goal.x[a] = int(v)
        # room for most programs; a longer one says how much it needs
        n = C.c_size_t(128)
        while True:
            cap = n.value
            nodes = (_ScheduleNode * cap)()
            rc = lib().mrl_schedule(self._h, C.byref(goal), nodes, C.c_size_t(cap), C.byref(n))
            if rc != E_BUFSZ or n.value <= cap:
                break
        _check(rc)
        dims = [len(t.extents) for t in self._schedule_tables()]
        return [(nd.table, tuple(nd.spec.x[:dims[nd.table]]), nd.rewrite, nd.cost, nd.n_children)
                for nd in nodes[:n.value]]

    def _schedule_tables(self):
        """Tables by the index a schedule node carries: this one, its deps, then the deps of its dep 1."""
        tabs = (self,) + tuple(self._deps)
        if len(self._deps) > 1:
            tabs += (None,) * (3 - len(tabs)) + tuple(self._deps[1]._deps)
        return tabs

    def program_text(self, coord):
        """The program of `coord` as indented text, one rewrite per line (the nesting of Section 2,
        Figure 1: a Move or a loop encloses the Spec it leaves, a microkernel is a leaf)."""
        tabs = self._schedule_tables()
        lines, open_children = [], []
        for t, x, rid, cost, k in self.schedule(coord):
            tab = tabs[t]
            sizes = tab.lattice["sizes"]
            r = tab.rewrite_decode(rid)
            if r.cls == 0:
                what = "microkernel %d" % r.mk_index
            elif r.cls == 1:
                what = "move operand %d to level %d%s%s" % (r.operand_or_dim, r.dst_level,
                                                           ", transposed" if r.transposed else "",
                                                           ", converted" if r.convert else "")
            elif r.cls == 2:
                d = r.operand_or_dim
                what = "loop over %s: %d steps of %d" % ("bmkn"[d], sizes[d][x[d]] // r.tile_size, r.tile_size)
            elif r.cls == 4:
                d = r.operand_or_dim
                what = "parallel loop over %s: %d steps of %d, serial-only body" % (
                    "bmkn"[d], sizes[d][x[d]] // r.tile_size, r.tile_size)
            else:
                what = "bufferize: the first stage into the intermediate, then the second out of it"
            lines.append("%stable %d  %s  %s  cost %d  %s" % ("  " * len(open_children), t,
                         "x".join(str(sizes[d][x[d]]) for d in range(4)), tuple(x[4:]), cost, what))
            if k:
                open_children.append(k)
            else:
                while open_children:
                    open_children[-1] -= 1
                    if open_children[-1]:
                        break
                    open_children.pop()
        return "\n".join(lines)

    def rewrite_decode(self, rid):
        r = Rewrite()
        _check(lib().mrl_rewrite_decode(self._h, C.c_uint16(rid), C.byref(r)))
        return r

    def coord_of_spec(self, shape, levels, layouts=None, dtypes=None):
        sh = (C.c_uint32 * 4)(*shape)
        lv = (C.c_uint8 * 5)(*(list(levels) + [0] * (5 - len(levels))))
        ly = (C.c_uint8 * 5)(*(list(layouts or []) + [0] * (5 - len(layouts or []))))
        dt = (C.c_uint8 * 5)(*(list(dtypes or []) + [0] * (5 - len(dtypes or []))))
        out = _Coord()
        _check(lib().mrl_coord_of_spec(self._h, sh, lv, ly, dt, C.byref(out)))
        return list(out.x[:len(self.extents)])

    def apply(self, coord, lhs, rhs, bias=None, out=None, workspace=None):
        """The operator of the Spec at `coord` on torch tensors of its sizes, layouts and types: a FUSED
        Spec gives relu(lhs rhs + bias), a Matmul lhs rhs, added to `out` if that is given.  Runs
        binding.linear; the program that the table found for the Spec is not what is run."""
        x = _Coord()
        for a, v in enumerate(coord):
            x.x[a] = int(v)
        raw = C.create_string_buffer(_LINEAR.size)
        _check(lib().mrl_spec_linear(self._h, C.byref(x), raw))
        spec = _LINEAR.unpack(raw.raw)
        b, m, k, n = spec[:4]
        codes = _dtype_codes()
        for name, t, at, shape in (("lhs", lhs, 4, (b, m, k)), ("rhs", rhs, 9, (b, k, n))):
            if tuple(t.shape) not in (shape, shape[1:] if b == 1 else shape):
                raise MorelloError(E_INVAL, "%s has shape %s, the Spec's is %s" % (name, tuple(t.shape), shape))
            if codes.get(t.dtype) != spec[at + 1]:
                raise MorelloError(E_INVAL, "%s is %s, the Spec's is another type" % (name, t.dtype))
            if min(shape[1:]) > 1 and _matrix(name, t)[2] != spec[at + 2]:
                raise MorelloError(E_INVAL, "%s has another layout than the Spec's" % name)
        fused = spec[17] != 0                    # the bias's stride
        if fused == (bias is None):
            raise MorelloError(E_INVAL, "a FUSED Spec takes a bias, a Matmul none")
        if fused and codes.get(bias.dtype) != spec[15]:
            raise MorelloError(E_INVAL, "bias is %s, the Spec's is another type" % bias.dtype)
        dtype = next(d for d, c in codes.items() if c == spec[25])
        return linear(lhs, rhs, bias, None if fused else out, activation="relu" if fused else "none", dtype=dtype,
                      out=out, workspace=workspace)

    def boxes(self, which):
        """which: 0 decisions, 1 costs.  numpy structured array (BOX_DTYPE), sorted by lo."""
        n = C.c_size_t()
        _check(lib().mrl_emit_compressed(self._h, C.c_uint32(which), None, C.c_size_t(0), C.byref(n)))
        out = np.zeros(n.value, dtype=BOX_DTYPE)
        _check(lib().mrl_emit_compressed(self._h, C.c_uint32(which), C.c_void_p(out.ctypes.data),
                                         C.c_size_t(n.value), C.byref(n)))
        return out

    def dense(self):
        cost = np.empty(self.n_specs, dtype=np.uint64)
        arg = np.empty(self.n_specs, dtype=np.uint16)
        _check(lib().mrl_copy_dense(self._h, cost.ctypes.data_as(C.POINTER(C.c_uint64)),
                                    arg.ctypes.data_as(C.POINTER(C.c_uint16))))
        return cost, arg


def solve(target, lattice, deps=(), scratch_bytes=None, stream=None, buffers=None):
    """Fill and compress one lattice on the current CUDA/HIP device.

    target: Target; lattice: dict (workloads.py); deps: solved Tables a fused
    lattice reads.  buffers: optional (cost, argmin, scratch) torch uint8
    tensors to reuse.  Device memory comes from torch; nothing else does.
    """
    import torch
    if not torch.cuda.is_available():
        raise RuntimeError("mrl solve needs a GPU: there is no CPU path")
    L = _lattice_desc(lattice)
    ext, n = geometry(target, lattice, desc=L)
    cb, ab = 8 * n, 2 * n
    if buffers is None:
        sb = table_bytes(target, lattice)[2] if scratch_bytes is None else scratch_bytes
        dev = torch.device("cuda", torch.cuda.current_device())
        buffers = (torch.empty(cb, dtype=torch.uint8, device=dev),
                   torch.empty(ab, dtype=torch.uint8, device=dev),
                   torch.empty(sb, dtype=torch.uint8, device=dev))
    d_cost, d_arg, d_scr = buffers
    assert d_cost.numel() >= cb and d_arg.numel() >= ab
    st = torch.cuda.current_stream() if stream is None else stream
    dep_arr = (C.c_void_p * max(1, len(deps)))(*[d._h for d in deps])
    h = C.c_void_p()
    stats = Stats()
    rc = lib().mrl_solve(target._h, C.byref(L), dep_arr if deps else None, C.c_uint32(len(deps)),
                         C.c_void_p(d_cost.data_ptr()), C.c_void_p(d_arg.data_ptr()),
                         C.c_void_p(d_scr.data_ptr()), C.c_size_t(d_scr.numel()),
                         C.c_void_p(st.cuda_stream), C.byref(h), C.byref(stats))
    _check(rc)
    return Table(h, target, lattice, ext, buffers, stats, deps)


_side_streams = {}


def _side_stream(dev, i):
    """The i-th extra stream of a device for the calling thread (default priority), created once."""
    import threading
    import torch
    pool = _side_streams.setdefault((dev, threading.get_ident()), [])
    while len(pool) <= i:
        pool.append(torch.cuda.Stream(device=dev))
    return pool[i]


class _Job(C.Structure):
    _fields_ = [("lattice", C.c_void_p), ("n_deps", C.c_uint32), ("deps", C.c_uint32 * 2),
                ("d_cost", C.c_void_p), ("d_argmin", C.c_void_p), ("d_scratch", C.c_void_p),
                ("scratch_bytes", C.c_size_t), ("hip_stream", C.c_void_p)]


def solve_lattices(target, lattices, scratch_bytes=None, buffers=None):
    """Solve [(label, lattice, dep labels)] with one call of mrl_solve_graph; returns {label: Table}.

    The library runs every lattice from a host thread of its own, on a stream of its own
    (default priority): lattices that do not depend on each other overlap on the device, and a
    lattice starts when the fill of those it reads is queued, while they are still being
    compressed.  buffers: optional {label: (cost, argmin, scratch)} torch uint8 tensors to reuse.
    """
    # dependency order (checked before any device work)
    order, seen, left = [], set(), list(lattices)
    while left:
        ok = [job for job in left if all(d in seen for d in job[2])]
        if not ok:
            raise ValueError("lattice dependencies form a cycle or name an unknown label")
        order += ok
        seen.update(job[0] for job in ok)
        left = [job for job in left if job[0] not in seen]
    import torch
    if not torch.cuda.is_available():
        raise RuntimeError("mrl solve needs a GPU: there is no CPU path")
    dev = torch.cuda.current_device()
    device = torch.device("cuda", dev)
    index = {job[0]: i for i, job in enumerate(order)}
    jobs = (_Job * len(order))()
    keep, held, exts = [], [], []
    for i, (label, lat, deps) in enumerate(order):
        L = _lattice_desc(lat)
        keep.append(L)
        ext, n = geometry(target, lat, desc=L)
        exts.append(ext)
        if buffers is None:
            sb = table_bytes(target, lat)[2] if scratch_bytes is None else scratch_bytes
            bufs = (torch.empty(8 * n, dtype=torch.uint8, device=device),
                    torch.empty(2 * n, dtype=torch.uint8, device=device),
                    torch.empty(sb, dtype=torch.uint8, device=device))
        else:
            bufs = buffers[label]
        assert bufs[0].numel() >= 8 * n and bufs[1].numel() >= 2 * n
        held.append(bufs)
        jobs[i].lattice = C.cast(C.pointer(L), C.c_void_p)
        jobs[i].n_deps = len(deps)
        for k, d in enumerate(deps):
            jobs[i].deps[k] = index[d]
        jobs[i].d_cost, jobs[i].d_argmin, jobs[i].d_scratch = (b.data_ptr() for b in bufs)
        jobs[i].scratch_bytes = bufs[2].numel()
        # the last lattice (on the calling thread) takes the current stream, the others side streams
        last = i == len(order) - 1
        jobs[i].hip_stream = torch.cuda.current_stream().cuda_stream if last else _side_stream(dev, i).cuda_stream
    handles = (C.c_void_p * len(order))()
    stats = (Stats * len(order))()
    torch.cuda.synchronize()            # the side streams start after everything queued so far
    _check(lib().mrl_solve_graph(target._h, jobs, C.c_uint32(len(order)), handles, stats))
    done = {}
    for i, (label, lat, deps) in enumerate(order):
        st = Stats.from_buffer_copy(stats[i])
        done[label] = Table(C.c_void_p(handles[i]), target, lat, exts[i], held[i], st, [done[d] for d in deps])
    return done


def solve_config(cfg, scratch_bytes=None):
    """Solve every lattice of a workloads.config() dict.  Returns (Target, {label: Table})."""
    target = Target(cfg["target"])
    return target, solve_lattices(target, cfg["lattices"], scratch_bytes=scratch_bytes)


# ---- the operators on torch tensors: the Matmul that Specs name, and what a layer made of it needs besides

ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}

# the C structs: b, m, k, n, then matrices of (data, dtype, layout, ld, batch), then what the operator adds
_LINEAR = struct.Struct("=4I" + "QIIqq" * 6 + "2I2Q")
_LINEAR_GRAD = struct.Struct("=4I" + "QIIqq" * 7 + "2I2Q")
_DROPOUT = struct.Struct("=2I" + "QIIqq" * 3 + "I4x2Q")
_NORM = struct.Struct("=3If" + "QIIqq" * 4 + "Q")
_NORM_GRAD = struct.Struct("=4I" + "QIIqq" * 7 + "Q")
_MX = struct.Struct("=4I" + "QIIqq" + "QQII")
_MX_LINEAR = struct.Struct("=4I" + "QIIqq" + "QQII" * 2 + "QIIqq" * 3 + "2I")
_ABSENT = (0, 0, 0, 0, 0)
_codes = _uint8 = _float32 = _empty_like = None


def _dtype_codes():
    global _codes, _uint8, _float32, _empty_like
    if _codes is None:
        import torch
        _codes, _uint8, _float32, _empty_like = {torch.float32: 0, torch.bfloat16: 1}, torch.uint8, torch.float32, torch.empty_like
    return _codes


def _dtype(name, t):
    code = (_codes or _dtype_codes()).get(t.dtype)
    if code is None:
        raise MorelloError(E_INVAL, "%s is %s: float32 and bfloat16 are what there is" % (name, t.dtype))
    return code


def _matrix(name, t):
    """(data, dtype, layout, ld, batch) of a tensor of two or three dimensions, either layout."""
    st, sh = t.stride(), t.shape
    if len(sh) == 2:
        (r, c), (rows, columns), batch = st, sh, 0
    elif len(sh) == 3:
        batch, r, c = st
        _, rows, columns = sh
    else:
        raise MorelloError(E_INVAL, "%s has %d dimensions: two, or three with a batch" % (name, len(sh)))
    if c == 1 and not (columns == 1 and r == 1):
        layout, ld = 0, r
    elif r == 1:
        layout, ld = 1, c
    elif columns <= 1:
        layout, ld = 0, r
    elif rows <= 1:
        layout, ld = 1, c
    else:
        raise MorelloError(E_INVAL, "%s: neither the elements of a row nor those of a column are adjacent (strides %s)" % (name, st))
    return t.data_ptr(), _dtype(name, t), layout, ld, batch


def _rows(name, t, shape):
    """The same of a row-major tensor of this shape."""
    if t.shape != shape:
        raise MorelloError(E_INVAL, "%s has shape %s, not %s" % (name, tuple(t.shape), tuple(shape)))
    st = t.stride()
    if st[-1] != 1 and shape[-1] > 1:
        raise MorelloError(E_INVAL, "%s: the elements of a row are not adjacent (strides %s)" % (name, st))
    return t.data_ptr(), _dtype(name, t), 0, st[-2], st[0] if len(st) == 3 else 0


def _vector(name, t, n):
    if t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise MorelloError(E_INVAL, "%s has shape %s and strides %s, not %d neighbouring elements" % (name, tuple(t.shape), t.stride(), n))
    return t.data_ptr(), _dtype(name, t), 0, 1, 0


def drop_threshold(p):
    """The `drop` of a probability: the nearest multiple of 2^-16, times 2^16."""
    if not 0.0 <= p <= 1.0:
        raise MorelloError(E_INVAL, "dropout of %r is no probability" % (p,))
    return int(p * 65536 + 0.5)


def _activation(name):
    if name not in ACTIVATIONS:
        raise MorelloError(E_INVAL, "activation %r is not one of %s" % (name, ", ".join(ACTIVATIONS)))
    return ACTIVATIONS[name]


def _word(name, v):
    if not 0 <= v < 1 << 64:
        raise MorelloError(E_INVAL, "%s %r does not fit 64 bits" % (name, v))
    return v


class _On:
    """Device and stream of a call that are not the current ones: with `stream` the outputs and the workspace belong
    to that stream, and torch is told that it uses the inputs (the caller orders it after whatever makes them)."""

    def __init__(self, index, tensors, stream):
        import torch
        if stream is None:
            self._within = torch.cuda.device(index)
            return
        if stream.device.index != index:
            raise MorelloError(E_INVAL, "the stream is on %s, the tensors on cuda:%d" % (stream.device, index))
        self._within = torch.cuda.stream(stream)
        for t in tensors:
            if t is not None:
                t.record_stream(stream)

    def __enter__(self):
        self._within.__enter__()

    def __exit__(self, *what):
        self._within.__exit__(*what)


_raw_stream = _current_device = None


def _elsewhere(tensors, stream):
    """Checks that all tensors (None: not given) are on one GPU.  Returns None where that is the current device and no stream
    is given, else the _On to be entered."""
    global _raw_stream, _current_device
    if _raw_stream is None:
        import torch
        # (what torch's own generated code asks; torch.cuda.current_stream makes a Stream object first, 1 us)
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    index = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise MorelloError(E_INVAL, "tensors on %s and %s" % (tensors[0].device, t.device))
    if index < 0:
        raise MorelloError(E_INVAL, "tensors on %s: there is no CPU path" % tensors[0].device)
    if stream is None and index == _current_device():
        return None
    return _On(index, tensors, stream)


def _run(desc, run, need, given, like):
    """Queue a call on the current stream; a workspace of torch's may be freed when this returns (work on its stream
    that uses the memory next comes after the call's)."""
    stream = _raw_stream(like.get_device())
    if need == 0:
        rc = run(desc, None, 0, stream)
    else:
        if given is None:
            given = like.new_empty(need, dtype=_uint8)
        elif not given.is_contiguous():
            raise MorelloError(E_INVAL, "the workspace is not contiguous")
        rc = run(desc, given.data_ptr(), given.numel() * given.element_size(), stream)
    if rc:
        _check(rc)


# What a call of linear or linear_grad with these sizes, strides, types and alignments comes to (no addresses, no values), worked
# out once: that takes 3 us of a call's 10.  As many as a program with many layers has.  (Of an address only whether it is a multiple of 16
# counts, of each operand by itself: one that is not may be copied into the workspace.  Of a probability its value now: it may come as an
# object that changes.)
_FORMS_MOST = 1024
_WORD_END = 1 << 64
_forms = {}


def _keep_form(key, form):
    if len(_forms) >= _FORMS_MOST:
        _forms.clear()
    _forms[key] = form
    return form


def _like(rhs, layout):
    """A tensor without gaps of rhs's shape and layout."""
    if layout:
        return rhs.new_empty(rhs.shape[:-2] + (rhs.shape[-1], rhs.shape[-2])).transpose(-1, -2)
    return rhs.new_empty(rhs.shape)


def _form_grad(key, grad, lhs, rhs, bias, pre, activation, drop, need_lhs, need_rhs):
    sizes, ml, mr, shape = _operands(lhs, rhs)
    act = _activation(activation)
    if act and pre is None:
        raise MorelloError(E_INVAL, "the gradient of %s needs pre" % activation)
    m_lhs = m_rhs = _ABSENT
    if need_lhs:
        m_lhs = _rows("d_lhs", lhs.new_empty(lhs.shape), lhs.shape)
    if need_rhs:                # (of one row or column d_rhs could be read either way: its layout is rhs's)
        d_rhs = _like(rhs, mr[2])
        st = d_rhs.stride()
        m_rhs = (d_rhs.data_ptr(), mr[1], mr[2], st[-1] if mr[2] else st[-2], st[0] if len(st) == 3 else 0)
    mats = [_rows("grad", grad, shape), ml, mr, _rows("pre", pre, shape) if act else _ABSENT, m_lhs, m_rhs,
            _ABSENT if bias is None else _vector("bias", bias, sizes[3])]
    n = C.c_size_t()
    _check(lib().mrl_linear_grad_bytes(_LINEAR_GRAD.pack(*sizes, *(v for m in mats for v in m), act, drop, 0, 0), C.addressof(n)))
    return _keep_form(key, (sizes, *(m[1:] for m in mats), act, n.value))


def _form_linear(key, lhs, rhs, bias, residual, out, dtype, pre, activation, drop):
    sizes, ml, mr, shape = _operands(lhs, rhs)
    if out is None:
        out = lhs.new_empty(shape, dtype=lhs.dtype if dtype is None else dtype)
    elif dtype is not None and out.dtype != dtype:
        raise MorelloError(E_INVAL, "out is %s, not %s" % (out.dtype, dtype))
    z = out.new_empty(shape) if pre else None
    mats = [ml, mr, _ABSENT if bias is None else _vector("bias", bias, sizes[3]), _ABSENT if residual is None else _rows("residual", residual, shape),
            _rows("out", out, shape), _ABSENT if z is None else _rows("pre", z, shape)]
    act = _activation(activation)
    n = C.c_size_t()
    _check(lib().mrl_linear_bytes(_LINEAR.pack(*sizes, *(v for m in mats for v in m), act, drop, 0, 0), C.addressof(n)))
    return _keep_form(key, (shape, out.dtype, sizes, *(m[1:] for m in mats), act, n.value))


def _operands(lhs, rhs):
    """(b, m, k, n), the two matrices and out's shape; rhs without a batch is shared by lhs's batches."""
    ml, mr = _matrix("lhs", lhs), _matrix("rhs", rhs)
    ls, rs = lhs.shape, rhs.shape
    if ls[-1] != rs[-2] or (len(rs) == 3 and (len(ls) != 3 or ls[0] != rs[0])):
        raise MorelloError(E_INVAL, "lhs of shape %s does not go with rhs of shape %s" % (tuple(ls), tuple(rs)))
    if len(ls) == 2:
        return (1, ls[0], ls[1], rs[-1]), ml, mr, (ls[0], rs[-1])
    return (ls[0], ls[1], ls[2], rs[-1]), ml, mr, (ls[0], ls[1], rs[-1])


def linear(lhs, rhs, bias=None, residual=None, *, activation="none", dropout=0.0, seed=0, offset=0, dtype=None, pre=False,
           out=None, workspace=None, stream=None):
    """out = residual + D f(lhs rhs + bias) (mrl_linear); with pre=True also z = lhs rhs + bias: (out, z).

    lhs: m x k or b x m x k, rhs: k x n or b x k x n, both float32 or both bfloat16, either one row- or
    column-major with any stride between lines (a weight matrix stored n x k is given as its .t()).
    bias: n elements; residual: of out's shape.  activation: none, relu, gelu (tanh form), silu.
    dropout: the probability that an element is dropped; seed and offset (64 bits each) say which are, together with
    the element's row and column.  dtype: out's and z's type (lhs's if None); out: a tensor to write to, which may be
    `residual`.  workspace: device memory that the caller keeps, a contiguous tensor (one that is too small is refused
    with E_NOMEM and what is needed); stream: where the work is queued (the current stream if None).  Autograd
    does not record the call: linear_grad is its gradient.
    """
    on = _elsewhere((lhs, rhs, bias, residual, out, workspace), stream)
    if on is not None:
        with on:
            return linear(lhs, rhs, bias, residual, activation=activation, dropout=dropout, seed=seed, offset=offset, dtype=dtype, pre=pre,
                          out=out, workspace=workspace)
    pl, pr, drop = lhs.data_ptr(), rhs.data_ptr(), drop_threshold(dropout)
    key = (lhs.shape, lhs.stride(), lhs.dtype, rhs.shape, rhs.stride(), rhs.dtype, pl & 15 == 0, pr & 15 == 0,
           None if bias is None else (bias.shape, bias.stride(), bias.dtype),
           None if residual is None else (residual.shape, residual.stride(), residual.dtype),
           None if out is None else (out.shape, out.stride(), out.dtype), dtype, pre, activation, drop)
    form = _forms.get(key)
    if form is None:
        form = _form_linear(key, lhs, rhs, bias, residual, out, dtype, pre, activation, drop)
    shape, dtype, sizes, ml, mr, mb, ms, mo, mz, act, need = form
    if out is None:
        out = lhs.new_empty(shape, dtype=dtype)
    z = out.new_empty(shape) if pre else None
    if not (0 <= seed < _WORD_END and 0 <= offset < _WORD_END):
        raise MorelloError(E_INVAL, "seed %r or offset %r does not fit 64 bits" % (seed, offset))
    desc = _LINEAR.pack(*sizes, pl, *ml, pr, *mr, 0 if bias is None else bias.data_ptr(), *mb, 0 if residual is None else residual.data_ptr(), *ms,
                        out.data_ptr(), *mo, z.data_ptr() if pre else 0, *mz, act, drop, seed, offset)
    _run(desc, _lib.mrl_linear, need, workspace, lhs)
    return (out, z) if pre else out


def linear_grad(grad, lhs, rhs, bias=None, pre=None, *, activation="none", dropout=0.0, seed=0, offset=0, need_lhs=True,
                need_rhs=True, workspace=None, stream=None):
    """(d_lhs, d_rhs, d_bias) of binding.linear with these arguments, given `grad`, the gradient by its out, and
    `pre`, the z that it returned (not needed without an activation): mrl_linear_grad.  Each has its operand's type,
    d_rhs also its layout; None for an operand that is not needed, or a bias that is None.  The gradient
    by the residual is `grad`."""
    on = _elsewhere((lhs, grad, rhs, bias, pre, workspace), stream)
    if on is not None:
        with on:
            return linear_grad(grad, lhs, rhs, bias, pre, activation=activation, dropout=dropout, seed=seed, offset=offset,
                               need_lhs=need_lhs, need_rhs=need_rhs, workspace=workspace)
    pg, pl, pr, drop = grad.data_ptr(), lhs.data_ptr(), rhs.data_ptr(), drop_threshold(dropout)
    key = (grad.shape, grad.stride(), grad.dtype, lhs.shape, lhs.stride(), lhs.dtype, rhs.shape, rhs.stride(), rhs.dtype, pg & 15 == 0, pl & 15 == 0, pr & 15 == 0,
           None if bias is None else (bias.shape, bias.stride(), bias.dtype), None if pre is None else (pre.shape, pre.stride(), pre.dtype),
           activation, drop, need_lhs, need_rhs)
    form = _forms.get(key)
    if form is None:
        form = _form_grad(key, grad, lhs, rhs, bias, pre, activation, drop, need_lhs, need_rhs)
    sizes, mg, ml, mr, mz, m_lhs, m_rhs, m_bias, act, need = form
    d_lhs = lhs.new_empty(lhs.shape) if need_lhs else None
    d_rhs = _like(rhs, mr[1]) if need_rhs else None
    d_bias = bias.new_empty(bias.shape) if bias is not None else None
    if not (0 <= seed < _WORD_END and 0 <= offset < _WORD_END):
        raise MorelloError(E_INVAL, "seed %r or offset %r does not fit 64 bits" % (seed, offset))
    desc = _LINEAR_GRAD.pack(*sizes, pg, *mg, pl, *ml, pr, *mr, pre.data_ptr() if act else 0, *mz, d_lhs.data_ptr() if need_lhs else 0, *m_lhs,
                             d_rhs.data_ptr() if need_rhs else 0, *m_rhs, 0 if bias is None else d_bias.data_ptr(), *m_bias, act, drop, seed, offset)
    _run(desc, _lib.mrl_linear_grad, need, workspace, lhs)
    return d_lhs, d_rhs, d_bias


def dropout(x, residual=None, *, dropout, seed=0, offset=0, out=None, stream=None):
    """residual + D x (mrl_dropout): x of m x n or b x m x n, rows without gaps between batches; see linear for the
    other arguments."""
    if x.dim() not in (2, 3):
        raise MorelloError(E_INVAL, "x has %d dimensions: two, or three with a batch" % x.dim())
    on = _elsewhere((x, residual, out), stream)
    if on is not None:
        with on:
            return _dropout(x, residual, dropout=dropout, seed=seed, offset=offset, out=out)
    if out is None:
        out = x.new_empty(x.shape)
    matrices = []
    for name, t in (("x", x), ("residual", residual), ("out", out)):
        if t is None:
            matrices += _ABSENT
            continue
        at = _rows(name, t, x.shape)
        if x.dim() == 3 and x.shape[0] > 1:
            if x.shape[1] <= 1:          # (a batch's only row has a stride that says nothing)
                at = at[:3] + (at[4], at[4])
            elif at[4] != x.shape[1] * at[3]:
                raise MorelloError(E_INVAL, "%s: its batches do not follow each other (strides %s)" % (name, t.stride()))
        matrices += at
    rows = x.shape[0] * x.shape[1] if x.dim() == 3 else x.shape[0]
    desc = _DROPOUT.pack(rows, x.shape[-1], *matrices, drop_threshold(dropout), _word("seed", seed), _word("offset", offset))
    rc = lib().mrl_dropout(desc, _raw_stream(x.get_device()))
    if rc:
        _check(rc)
    return out


def dropout_grad(grad, *, dropout, seed=0, offset=0, out=None, stream=None):
    """The gradient of binding.dropout by x, given `grad`, that by its result: D grad."""
    return _dropout(grad, dropout=dropout, seed=seed, offset=offset, out=out, stream=stream)


_dropout = dropout


def _rows_count(name, t):
    """(b, m, n) of a tensor of rows."""
    sh = t.shape
    if len(sh) == 2:
        return 1, sh[0], sh[1]
    if len(sh) == 3:
        return tuple(sh)
    raise MorelloError(E_INVAL, "%s has %d dimensions: two, or three with a batch" % (name, len(sh)))


def _of(t):
    return None if t is None else (t.shape, t.stride(), t.dtype)


def _form_norm(key, x, weight, bias, dtype, out):
    sizes = _rows_count("x", x)
    if out is None:
        out = x.new_empty(x.shape, dtype=x.dtype if dtype is None else dtype)
    elif dtype is not None and out.dtype != dtype:
        raise MorelloError(E_INVAL, "out is %s, not %s" % (out.dtype, dtype))
    mats = [_rows("x", x, x.shape), _rows("out", out, x.shape)]
    for name, v in (("weight", weight), ("bias", bias)):
        mats.append(_ABSENT if v is None else _vector(name, v, sizes[2]))
    return _keep_form(key, (sizes, *(m[1:] for m in mats), out.dtype, x.is_contiguous() and out.dtype == x.dtype))


def layer_norm(x, weight=None, bias=None, *, eps=1e-5, stats=False, dtype=None, out=None, stream=None):
    """(x - mean) r weight + bias over the last dimension, r = 1 / sqrt(variance + eps) (mrl_layer_norm); with stats=True
    also (mean, r) of every row, float32 of x's leading dimensions by 2, which layer_norm_grad needs: (out, stats).  Rows of no elements have NaN there.

    x: m x n or b x m x n, rows at any stride; weight, bias: n elements, 1 and 0 if None; each float32 or bfloat16.
    dtype: out's type (x's if None); out: a tensor to write to, which may be x itself; stream: as for linear."""
    on = _elsewhere((x, weight, bias, out), stream)
    if on is not None:
        with on:
            return layer_norm(x, weight, bias, eps=eps, stats=stats, dtype=dtype, out=out)
    key = ("norm", x.shape, x.stride(), x.dtype, _of(weight), _of(bias), _of(out), dtype)
    sizes, mx, mo, mw, mb, dtype, like = _forms.get(key) or _form_norm(key, x, weight, bias, dtype, out)
    if not 0.0 <= eps <= 3.4e38:
        raise MorelloError(E_INVAL, "eps of %r is negative or not finite" % (eps,))
    if out is None:              # (of a tensor without gaps the same again, which takes torch two thirds of the time)
        out = _empty_like(x) if like else x.new_empty(x.shape, dtype=dtype)
    kept = x.new_empty(x.shape[:-1] + (2,), dtype=_float32) if stats else None
    if stats and not sizes[2]:   # (the library writes nothing; there is no mean of nothing)
        kept.fill_(float("nan"))
    desc = _NORM.pack(*sizes, eps, x.data_ptr(), *mx, out.data_ptr(), *mo, 0 if weight is None else weight.data_ptr(), *mw,
                      0 if bias is None else bias.data_ptr(), *mb, kept.data_ptr() if stats else 0)
    rc = lib().mrl_layer_norm(desc, _raw_stream(x.get_device()))
    if rc:
        _check(rc)
    return (out, kept) if stats else out


def _form_norm_grad(key, grad, x, stats, weight, bias, residual, need_x):
    _dtype_codes()
    sizes = _rows_count("x", x)
    if stats.shape != x.shape[:-1] + (2,) or stats.dtype != _float32 or not stats.is_contiguous():
        raise MorelloError(E_INVAL, "stats of shape %s, %s: what layer_norm returns has shape %s, float32, without gaps" % (tuple(stats.shape), stats.dtype,
                                                                                                            tuple(x.shape[:-1]) + (2,)))
    mats = [_rows("grad", grad, x.shape), _rows("x", x, x.shape), _ABSENT if residual is None else _rows("residual", residual, x.shape),
            _ABSENT if weight is None else _vector("weight", weight, sizes[2]), _rows("d_x", x.new_empty(x.shape), x.shape) if need_x else _ABSENT]
    for name, v in (("weight", weight), ("bias", bias)):
        mats.append(_ABSENT if v is None else _vector(name, v, sizes[2]))
    desc = _NORM_GRAD.pack(*sizes, 0, *(v for m in mats for v in m), stats.data_ptr())
    n = C.c_size_t()
    _check(lib().mrl_layer_norm_grad_bytes(desc, C.addressof(n)))
    return _keep_form(key, (sizes, *(m[1:] for m in mats), n.value, x.is_contiguous()))


def layer_norm_grad(grad, x, stats, weight=None, bias=None, residual=None, *, need_x=True, workspace=None, stream=None):
    """(d_x, d_weight, d_bias) of layer_norm(x, weight, bias), given `grad`, the gradient by its out, and the
    `stats` that it returned (mrl_layer_norm_grad).  Each has its operand's type; None for d_x without need_x, and for a
    weight or bias that is None.  residual: the gradient that reaches x past the normalisation, added to
    d_x."""
    on = _elsewhere((x, grad, stats, weight, bias, residual, workspace), stream)
    if on is not None:
        with on:
            return layer_norm_grad(grad, x, stats, weight, bias, residual, need_x=need_x, workspace=workspace)
    key = ("norm_grad", grad.shape, grad.stride(), grad.dtype, x.shape, x.stride(), x.dtype, _of(stats), _of(weight), _of(bias), _of(residual), need_x)
    form = _forms.get(key)
    if form is None:
        form = _form_norm_grad(key, grad, x, stats, weight, bias, residual, need_x)
    sizes, mg, mx, mr, mw, m_x, m_weight, m_bias, need, like = form
    d_x = (_empty_like(x) if like else x.new_empty(x.shape)) if need_x else None
    d_weight = None if weight is None else _empty_like(weight)
    d_bias = None if bias is None else _empty_like(bias)
    desc = _NORM_GRAD.pack(*sizes, 0, grad.data_ptr(), *mg, x.data_ptr(), *mx, 0 if residual is None else residual.data_ptr(), *mr,
                           0 if weight is None else weight.data_ptr(), *mw, d_x.data_ptr() if need_x else 0, *m_x,
                           0 if weight is None else d_weight.data_ptr(), *m_weight, 0 if bias is None else d_bias.data_ptr(), *m_bias, stats.data_ptr())
    _run(desc, _lib.mrl_layer_norm_grad, need, workspace, x)
    return d_x, d_weight, d_bias


# ---- microscaled 4-bit floating point

class MX:
    """A tensor in blocks of 32 values along k: 4 bits a value and a byte of scale a block (the header at mrl_mx has the format).

    codes: uint8 of (batch,) lines x 64 ceil(k / 128); scales: uint8 of (batch,) ceil(lines / 64) x ceil(k / 128) x 4 x 16 x 4, both
    without gaps.  dim: the dimension that the blocks run along, -1 (the lines are rows: the tensor is lines x k) or -2 (they are
    columns: k x lines, as linear's rhs).  dtype: the type that the tensor had and is read back in.  The attributes of one that is made stay as they are
    (what a call comes to is kept by them); the tensors' elements may change."""
    __slots__ = ("codes", "scales", "k", "dim", "dtype", "shape", "_key")

    def __init__(self, codes, scales, k, *, dim=-1, dtype=None):
        if dtype is None:
            import torch
            dtype = torch.bfloat16
        # (worked out once for shapes: an MX may be made anew around the same tensors for every call)
        key = ("mx", codes.shape, scales.shape, codes.stride(), scales.stride(), codes.dtype, scales.dtype, k, dim, dtype)
        self.codes, self.scales, self.k, self.dim, self.dtype = codes, scales, k, dim, dtype
        self.shape, self._key = _forms.get(key) or _form_mx(key, codes, scales, k, dim, dtype)

    @property
    def lines(self):
        return self.codes.shape[-2]

    def __repr__(self):
        return "MX(shape=%s, dim=%d, dtype=%s)" % (tuple(self.shape), self.dim, self.dtype)


def _form_mx(key, codes, scales, k, dim, dtype):
    _dtype_codes()
    if dim not in (-1, -2):
        raise MorelloError(E_INVAL, "dim of %r: blocks run along the last dimension (-1) or the one before (-2)" % (dim,))
    if dtype not in _codes:
        raise MorelloError(E_INVAL, "%s: float32 and bfloat16 are what there is" % (dtype,))
    if codes.dtype != _uint8 or scales.dtype != _uint8 or not codes.is_contiguous() or not scales.is_contiguous():
        raise MorelloError(E_INVAL, "codes and scales are uint8 without gaps")
    if len(codes.shape) not in (2, 3) or not 0 <= k < 1 << 31:
        raise MorelloError(E_INVAL, "codes of shape %s: lines, or a batch of them" % (tuple(codes.shape),))
    lead, lines, steps = tuple(codes.shape[:-2]), codes.shape[-2], -(-k // 128)
    if codes.shape[-1] != 64 * steps or tuple(scales.shape) != lead + (-(-lines // 64), steps, 4, 16, 4):
        raise MorelloError(E_INVAL, "codes of shape %s and scales of shape %s are not those of %d lines of %d values" % (
            tuple(codes.shape), tuple(scales.shape), lines, k))
    shape = codes.shape[:-2] + ((lines, k) if dim == -1 else (k, lines))
    return _keep_form(key, (shape, (shape, dim, dtype)))


def mx_quantize(x, *, dim=-1, out=None, stream=None):
    """x in blocks of 32 values along `dim` (-1, or -2 as for linear's rhs): an MX (mrl_mx_quantize).  x: two dimensions, or three with a
    batch; float32 or bfloat16, row- or column-major with any stride between lines.  out: an MX of this shape and dim to write to."""
    on = _elsewhere((x,) if out is None else (x, out.codes, out.scales), stream)
    if on is not None:
        with on:
            return mx_quantize(x, dim=dim, out=out)
    key = ("mx_quantize", x.shape, x.stride(), x.dtype, dim)
    form = _forms.get(key)
    if form is None:
        b, _, _ = _rows_count("x", x)
        if dim not in (-1, -2):
            raise MorelloError(E_INVAL, "dim of %r: blocks run along the last dimension (-1) or the one before (-2)" % (dim,))
        # (lines along k: of x itself, or of its transpose)
        lines = x if dim == -1 else x.transpose(-1, -2)
        n, k = lines.shape[-2:]
        steps = -(-k // 128)
        codes, scales = lines.shape[:-2] + (n, 64 * steps), lines.shape[:-2] + (-(-n // 64), steps, 4, 16, 4)
        form = ((b, n, k, 0), _matrix("x", lines)[1:], codes, scales, MX(x.new_empty(codes, dtype=_uint8), x.new_empty(scales, dtype=_uint8), k, dim=dim, dtype=x.dtype)._key)
        _keep_form(key, form)
    sizes, m, codes, scales, kept = form
    if out is None:
        out = MX.__new__(MX)       # (its checks are the form's)
        out.codes, out.scales, out.k, out.dim, out.dtype = x.new_empty(codes, dtype=_uint8), x.new_empty(scales, dtype=_uint8), sizes[2], dim, x.dtype
        out.shape, out._key = x.shape, kept
    elif out.shape != x.shape or out.dim != dim:
        raise MorelloError(E_INVAL, "out is %r: x has shape %s, dim %d" % (out, tuple(x.shape), dim))
    rc = lib().mrl_mx_quantize(_MX.pack(*sizes, x.data_ptr(), *m, out.codes.data_ptr(), out.scales.data_ptr(), 0, 0), _raw_stream(x.get_device()))
    if rc:
        _check(rc)
    return out


def mx_dequantize(q, *, dtype=None, stream=None):
    """What an MX stands for, in q.dtype or `dtype`, both exact (mrl_mx_dequantize); with dim=-2 it comes column-major, as its lines are."""
    on = _elsewhere((q.codes, q.scales), stream)
    if on is not None:
        with on:
            return mx_dequantize(q, dtype=dtype)
    dtype = q.dtype if dtype is None else dtype
    key = ("mx_dequantize", q._key, dtype)
    form = _forms.get(key)
    if form is None:
        lead, lines, k = q.codes.shape[:-2], q.lines, q.k
        like = q.codes.new_empty(lead + (lines, k), dtype=dtype)
        form = _keep_form(key, (_rows_count("x", like) + (0,), lead + (lines, k), _rows("x", like, like.shape)[1:]))
    sizes, shape, m = form
    out = q.codes.new_empty(shape, dtype=dtype)
    rc = lib().mrl_mx_dequantize(_MX.pack(*sizes, out.data_ptr(), *m, q.codes.data_ptr(), q.scales.data_ptr(), 0, 0), _raw_stream(out.get_device()))
    if rc:
        _check(rc)
    return out if q.dim == -1 else out.transpose(-1, -2)


def _form_mx_linear(key, lhs, rhs, blocks, bias, residual, out, dtype, activation):
    if rhs.dim != -2 or (blocks and lhs.dim != -1):
        raise MorelloError(E_INVAL, "lhs is in blocks along its last dimension, rhs along the one before: %r, %r" % (lhs, rhs))
    ls, rs = lhs.shape, rhs.shape
    b, m, k = _rows_count("lhs", lhs)
    if k != rs[-2] or (len(rs) == 3 and (len(ls) != 3 or ls[0] != rs[0])):
        raise MorelloError(E_INVAL, "lhs of shape %s does not go with rhs of shape %s" % (tuple(ls), tuple(rs)))
    n = rs[-1]
    shape = ls[:-1] + (n,)
    like = lhs.codes if blocks else lhs
    if out is None:
        out = like.new_empty(shape, dtype=lhs.dtype if dtype is None else dtype)
    elif dtype is not None and out.dtype != dtype:
        raise MorelloError(E_INVAL, "out is %s, not %s" % (out.dtype, dtype))
    ml = _ABSENT if blocks else _matrix("lhs", lhs)
    mats = [_ABSENT if bias is None else _vector("bias", bias, n), _ABSENT if residual is None else _rows("residual", residual, shape), _rows("out", out, shape)]
    act = _activation(activation)
    sizes, shared = (b, m, k, n), int(len(rs) == 2)
    desc = _MX_LINEAR.pack(*sizes, *ml, *((like.data_ptr(), lhs.scales.data_ptr()) if blocks else (0, 0)), 0, 0, rhs.codes.data_ptr(), rhs.scales.data_ptr(), shared, 0,
                           *(v for m in mats for v in m), act, 0)
    need = C.c_size_t()
    _check(lib().mrl_mx_linear_bytes(desc, C.addressof(need)))
    return _keep_form(key, (shape, None if out.dtype == like.dtype else out.dtype, sizes, shared, ml[1:], *(m[1:] for m in mats), act, need.value))


def mx_linear(lhs, rhs, bias=None, residual=None, *, activation="none", dtype=None, out=None, workspace=None, stream=None):
    """out = residual + f(lhs rhs + bias) (mrl_mx_linear), as linear, of operands in blocks of 4-bit values.

    rhs: an MX of k x n or b x k x n with dim=-2 (mx_quantize(weight, dim=-2)); lhs: an MX of m x k or b x m x k with dim=-1, or a tensor,
    which the call quantises as mx_quantize does.  The other arguments are linear's; dtype: out's type (lhs's if None)."""
    blocks = type(lhs) is MX
    on = _elsewhere((lhs.codes if blocks else lhs, lhs.scales if blocks else None, rhs.codes, rhs.scales, bias, residual, out, workspace), stream)
    if on is not None:
        with on:
            return mx_linear(lhs, rhs, bias, residual, activation=activation, dtype=dtype, out=out, workspace=workspace)
    key = ("mx_linear", lhs._key if blocks else (lhs.shape, lhs.stride(), lhs.dtype), rhs._key, _of(bias), _of(residual), _of(out), dtype, activation)
    form = _forms.get(key)
    if form is None:
        form = _form_mx_linear(key, lhs, rhs, blocks, bias, residual, out, dtype, activation)
    shape, dtype, sizes, shared, ml, mb, ms, mo, act, need = form
    if blocks:
        like, first = lhs.codes, (0, *ml, lhs.codes.data_ptr(), lhs.scales.data_ptr())
    else:
        like, first = lhs, (lhs.data_ptr(), *ml, 0, 0)
    if out is None:
        out = like.new_empty(shape) if dtype is None else like.new_empty(shape, dtype=dtype)
    desc = _MX_LINEAR.pack(*sizes, *first, 0, 0, rhs.codes.data_ptr(), rhs.scales.data_ptr(), shared, 0, 0 if bias is None else bias.data_ptr(), *mb,
                           0 if residual is None else residual.data_ptr(), *ms, out.data_ptr(), *mo, act, 0)
    _run(desc, _lib.mrl_mx_linear, need, workspace, like)
    return out
