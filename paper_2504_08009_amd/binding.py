"""ctypes binding of liboz2.so.  Function names follow include/oz2.h; arguments are marshalled only."""
import ctypes
import os
import struct

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "liboz2.so")
_lib = None

SYMBOLS = [
    "oz2_init", "oz2_min_moduli", "oz2_moduli_for_bits", "oz2_max_moduli", "oz2_get_moduli", "oz2_workspace_bytes", "oz2_workspace_bytes_for", "oz2_set_workspace",
    "oz2_workspace_layout", "oz2_dgemm", "oz2_dgemm_static", "oz2_dgemm_ex", "oz2_dsyrk", "oz2_dtrmm", "oz2_stage1_convert", "oz2_stage2_gemm", "oz2_stage3_crt",
    "oz2_set_gemm_algorithm", "oz2_gemm_algorithm_for", "oz2_workspace_bytes_strassen", "oz2_workspace_bytes_preferred",
    "oz2_context_create", "oz2_context_destroy", "oz2_context_set_workspace", "oz2_context_set", "oz2_context_get",
    "oz2_context_workspace_bytes", "oz2_context_dgemm", "oz2_context_dsyrk", "oz2_context_dtrmm",
    "oz2_set_kblock", "oz2_set_round_sync", "oz2_set_shift_mode", "oz2_set_product_format", "oz2_set_bit_split", "oz2_set_nonfinite_check", "oz2_set_stage_events", "oz2_calibrate_mfma", "oz2_host_kernel_choice", "oz2_host_route", "oz2_host_crt_element", "oz2_host_crt_element_digits", "oz2_host_crt_element_wide_digits", "oz2_host_residues", "oz2_host_product_residues", "oz2_host_short_product_residues", "oz2_status_string",
    "oz2_w4_matvec", "oz2_w4_moe_workspace_bytes", "oz2_w4_moe", "oz2_context_w4_moe",
    "oz2_attention", "oz2_kv4_append", "oz2_kv4_attention_workspace_bytes", "oz2_kv4_attention", "oz2_context_kv4_attention",
    "oz2_kv4_evict_workspace_bytes", "oz2_kv4_evict", "oz2_context_kv4_evict",
]


class Oz2Error(RuntimeError):
    pass


def lib():
    """Load liboz2.so (built by paper_2504_08009_amd/build.py).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise Oz2Error("liboz2.so is missing: run `python -c 'import __graft_entry__ as g; g.build()'` first")
        L = ctypes.CDLL(_LIB_PATH)
        i64, vp, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
        L.oz2_get_moduli.argtypes = [ci, vp, vp, i64]
        L.oz2_moduli_for_bits.argtypes = [i64, ci]
        L.oz2_workspace_bytes.restype = ctypes.c_size_t
        L.oz2_workspace_bytes.argtypes = [i64, i64, i64, ci]
        L.oz2_workspace_bytes_for.restype = ctypes.c_size_t
        L.oz2_workspace_bytes_for.argtypes = [i64, i64, i64, ci, ci]
        L.oz2_workspace_bytes_strassen.restype = ctypes.c_size_t
        L.oz2_workspace_bytes_strassen.argtypes = [i64, i64, i64, ci]
        L.oz2_workspace_bytes_preferred.restype = ctypes.c_size_t
        L.oz2_workspace_bytes_preferred.argtypes = [i64, i64, i64, ci]
        L.oz2_set_gemm_algorithm.argtypes = [ci]
        L.oz2_gemm_algorithm_for.argtypes = [i64, i64, i64, ci]
        L.oz2_set_workspace.argtypes = [vp, ctypes.c_size_t]
        L.oz2_workspace_layout.argtypes = [i64, i64, i64, ci, vp, vp]
        L.oz2_dgemm.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, ci, vp]
        L.oz2_dgemm_static.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, ci, vp]
        L.oz2_dgemm_ex.argtypes = [ctypes.c_char, ctypes.c_char, i64, i64, i64, ctypes.c_double, vp, i64, vp, i64,
                                   ctypes.c_double, vp, i64, ci, vp]
        L.oz2_dsyrk.argtypes = [ctypes.c_char, ctypes.c_char, i64, i64, ctypes.c_double, vp, i64, ctypes.c_double, vp, i64,
                                ci, vp]
        L.oz2_dtrmm.argtypes = [ctypes.c_char] * 4 + [i64, i64, ctypes.c_double, vp, i64, vp, i64, ci, vp]
        L.oz2_stage1_convert.argtypes = [i64, i64, i64, vp, i64, vp, i64, ci, vp]
        L.oz2_stage2_gemm.argtypes = [i64, i64, i64, ci, vp]
        L.oz2_stage3_crt.argtypes = [i64, i64, i64, vp, i64, ci, vp]
        L.oz2_set_kblock.argtypes = [i64]
        L.oz2_context_create.argtypes = [vp]
        L.oz2_context_destroy.argtypes = [vp]
        L.oz2_context_set_workspace.argtypes = [vp, vp, ctypes.c_size_t]
        L.oz2_context_set.argtypes = [vp, ci, i64]
        L.oz2_context_get.argtypes = [vp, ci, vp]
        L.oz2_context_workspace_bytes.restype = ctypes.c_size_t
        L.oz2_context_workspace_bytes.argtypes = [vp, i64, i64, i64, ci]
        L.oz2_context_dgemm.argtypes = [vp, ctypes.c_char, ctypes.c_char, i64, i64, i64, ctypes.c_double, vp, i64, vp, i64,
                                        ctypes.c_double, vp, i64, ci, vp]
        L.oz2_context_dsyrk.argtypes = [vp, ctypes.c_char, ctypes.c_char, i64, i64, ctypes.c_double, vp, i64, ctypes.c_double,
                                        vp, i64, ci, vp]
        L.oz2_context_dtrmm.argtypes = [vp] + [ctypes.c_char] * 4 + [i64, i64, ctypes.c_double, vp, i64, vp, i64, ci, vp]
        L.oz2_set_round_sync.argtypes = [ci]
        L.oz2_set_shift_mode.argtypes = [ci]
        L.oz2_set_product_format.argtypes = [ci]
        L.oz2_set_nonfinite_check.argtypes = [ci]
        L.oz2_set_bit_split.argtypes = [ci]
        L.oz2_set_stage_events.argtypes = [vp]
        L.oz2_calibrate_mfma.argtypes = [ci, ci, ci, vp, vp, vp]
        L.oz2_host_crt_element.argtypes = [ci, vp, vp]
        L.oz2_host_crt_element_digits.argtypes = [ci, vp, vp]
        L.oz2_host_crt_element_wide_digits.argtypes = [ci, vp, vp]
        L.oz2_host_kernel_choice.argtypes = [ci, i64, i64, i64, ci, ci, vp]
        L.oz2_host_route.argtypes = [ci, ctypes.c_char, ctypes.c_char, i64, i64, i64, ci, ci, vp]
        L.oz2_host_residues.argtypes = [ci, ci, ctypes.c_double, ci, vp]
        L.oz2_host_product_residues.argtypes = [ci, i64, vp, vp]
        L.oz2_host_short_product_residues.argtypes = [ci, i64, vp, vp]
        cf = ctypes.c_float
        L.oz2_w4_matvec.argtypes = [vp, i64, cf, ci, vp, i64, cf, vp, i64, ci, vp, i64, vp]
        L.oz2_w4_moe_workspace_bytes.restype = ctypes.c_size_t
        L.oz2_w4_moe_workspace_bytes.argtypes = [vp, i64]
        L.oz2_w4_moe.argtypes = [vp, i64, ci, vp, i64, vp, ci, vp, i64, vp, vp, vp]
        L.oz2_context_w4_moe.argtypes = [vp, vp, i64, ci, vp, i64, vp, ci, vp, i64, vp, vp, vp]
        L.oz2_attention.argtypes = [i64, i64, vp, i64, i64, i64, cf, ci, vp, vp, vp, vp, vp]
        L.oz2_kv4_append.argtypes = [vp, vp, vp, vp, vp, vp, vp, vp]
        L.oz2_kv4_attention_workspace_bytes.restype = ctypes.c_size_t
        L.oz2_kv4_attention_workspace_bytes.argtypes = [vp, i64, i64, i64, i64, ci]
        L.oz2_kv4_attention.argtypes = [vp, vp, i64, cf, vp, vp, vp]
        L.oz2_context_kv4_attention.argtypes = [vp, vp, vp, i64, cf, vp, vp, vp]
        L.oz2_kv4_evict_workspace_bytes.restype = ctypes.c_size_t
        L.oz2_kv4_evict_workspace_bytes.argtypes = [vp, i64, i64, i64]
        L.oz2_kv4_evict.argtypes = [vp, vp, i64, i64, vp, vp]
        L.oz2_context_kv4_evict.argtypes = [vp, vp, vp, i64, i64, vp, vp]
        L.oz2_status_string.restype = ctypes.c_char_p
        L.oz2_status_string.argtypes = [ci]
        _lib = L
    return _lib


def _check(rc, what):
    if rc != 0:
        raise Oz2Error("%s failed: status %d (%s)" % (what, rc, lib().oz2_status_string(rc).decode()))


def min_moduli():
    return lib().oz2_min_moduli()


def max_moduli():
    return lib().oz2_max_moduli()


def get_moduli(num_moduli, k=1):
    """(moduli list, kappa) for this moduli count and inner dimension."""
    mods = (ctypes.c_int * num_moduli)()
    kap = ctypes.c_int(0)
    _check(lib().oz2_get_moduli(num_moduli, mods, ctypes.byref(kap), k), "oz2_get_moduli")
    return list(mods), kap.value


def workspace_bytes(m, n, k, num_moduli, product_format=None):
    """Bytes that serve either product format (None), or exactly one of them."""
    if product_format is None:
        return int(lib().oz2_workspace_bytes(m, n, k, num_moduli))
    return int(lib().oz2_workspace_bytes_for(m, n, k, num_moduli, int(product_format)))


def workspace_bytes_strassen(m, n, k, num_moduli):
    """Bytes the Strassen form of the products needs."""
    return int(lib().oz2_workspace_bytes_strassen(m, n, k, num_moduli))


def workspace_bytes_preferred(m, n, k, num_moduli):
    """Bytes with which a general product takes the form the settings in force prefer."""
    return int(lib().oz2_workspace_bytes_preferred(m, n, k, num_moduli))


OZ2_GEMM_AUTO, OZ2_GEMM_CLASSICAL, OZ2_GEMM_STRASSEN = -1, 0, 1


def oz2_set_gemm_algorithm(algorithm):
    """-1 (default): Strassen form for large general products; 0: never; 1: whenever it applies."""
    _check(lib().oz2_set_gemm_algorithm(int(algorithm)), "oz2_set_gemm_algorithm")


def oz2_gemm_algorithm_for(m, n, k, num_moduli):
    """Form (0 classical, 1 Strassen) a general product of this shape takes under the settings and workspace in force."""
    rc = lib().oz2_gemm_algorithm_for(m, n, k, num_moduli)
    if rc < 0:
        raise Oz2Error("oz2_gemm_algorithm_for: invalid argument %d" % -rc)
    return rc


def oz2_init():
    _check(lib().oz2_init(), "oz2_init")


def moduli_for_bits(k, bits=53):
    """Smallest number of moduli whose bit budget reaches `bits` for inner dimension k (0: none does)."""
    rc = lib().oz2_moduli_for_bits(int(k), int(bits))
    if rc < 0:
        raise Oz2Error("oz2_moduli_for_bits: invalid argument %d" % -rc)
    return rc


def workspace_layout(m, n, k, num_moduli):
    """dict of byte offsets and padded dims (see include/oz2.h)."""
    offs = (ctypes.c_size_t * 10)()
    dims = (ctypes.c_int64 * 3)()
    _check(lib().oz2_workspace_layout(m, n, k, num_moduli, offs, dims), "oz2_workspace_layout")
    names = ["rowmax", "colmax", "sa", "sb", "a_planes", "b_planes", "c_planes", "rownorm", "colnorm", "flags"]
    out = {nm: int(o) for nm, o in zip(names, offs)}
    out.update(m_pad=int(dims[0]), n_pad=int(dims[1]), k_pad=int(dims[2]))
    return out


_registered_ptr = None   # what this module last registered with the library (None: nothing)


def set_workspace(dev_ptr, nbytes):
    global _registered_ptr
    _check(lib().oz2_set_workspace(dev_ptr, nbytes), "oz2_set_workspace")
    _registered_ptr = dev_ptr if dev_ptr else None


def oz2_set_round_sync(spins):
    """Bound (in polls) of a wait of the GEMM's per-die round synchronisation; 0 switches it off (default 4096)."""
    _check(lib().oz2_set_round_sync(int(spins)), "oz2_set_round_sync")


def oz2_set_kblock(kblock):
    _check(lib().oz2_set_kblock(kblock), "oz2_set_kblock")


def oz2_set_shift_mode(mode):
    """0: shifts from maxima (Section 3); 1: Cauchy-Schwarz bound; 2: INT8-product bound (both Section 4.1)."""
    _check(lib().oz2_set_shift_mode(int(mode)), "oz2_set_shift_mode")


OZ2_SHIFT_MAX, OZ2_SHIFT_CAUCHY_SCHWARZ, OZ2_SHIFT_INT8_PRODUCT = 0, 1, 2
OZ2_PRODUCT_INT32, OZ2_PRODUCT_RESIDUE_U8 = 0, 1


def oz2_set_product_format(fmt):
    """0: INT32 products in the C planes; 1 (default): UINT8 residues written by the GEMM epilogue."""
    _check(lib().oz2_set_product_format(int(fmt)), "oz2_set_product_format")


def oz2_set_bit_split(delta):
    """Bits of budget moved from op(A) to op(B) (0: the equal split)."""
    _check(lib().oz2_set_bit_split(int(delta)), "oz2_set_bit_split")


def oz2_set_nonfinite_check(on):
    """1 (default): infinities / NaNs in A or B are detected and C is formed by the FP64 fallback kernel."""
    _check(lib().oz2_set_nonfinite_check(int(on)), "oz2_set_nonfinite_check")


def oz2_set_stage_events(events):
    """events: four hipEvent_t handles (ints) or None."""
    if events is None:
        _check(lib().oz2_set_stage_events(None), "oz2_set_stage_events")
    else:
        arr = (ctypes.c_void_p * 4)(*events)
        _check(lib().oz2_set_stage_events(arr), "oz2_set_stage_events")


def _stream_ptr(stream):
    if stream is None:
        import torch
        stream = torch.cuda.current_stream()
    return getattr(stream, "cuda_stream", stream)


def oz2_dgemm(m, n, k, A_ptr, lda, B_ptr, ldb, C_ptr, ldc, num_moduli, stream=None):
    _check(lib().oz2_dgemm(m, n, k, A_ptr, lda, B_ptr, ldb, C_ptr, ldc, num_moduli, _stream_ptr(stream)), "oz2_dgemm")


OZ2_STATIC_SCRATCH_BYTES = 64 << 20


def oz2_dgemm_static(m, n, k, A_ptr, lda, B_ptr, ldb, C_ptr, ldc, num_moduli, stream=None):
    """oz2_dgemm on the library's static workspace: allocates nothing, needs no registered workspace."""
    _check(lib().oz2_dgemm_static(m, n, k, A_ptr, lda, B_ptr, ldb, C_ptr, ldc, num_moduli, _stream_ptr(stream)),
           "oz2_dgemm_static")


def oz2_dgemm_ex(transa, transb, m, n, k, alpha, A_ptr, lda, B_ptr, ldb, beta, C_ptr, ldc, num_moduli, stream=None):
    _check(lib().oz2_dgemm_ex(transa.encode(), transb.encode(), m, n, k, float(alpha), A_ptr, lda, B_ptr, ldb,
                              float(beta), C_ptr, ldc, num_moduli, _stream_ptr(stream)), "oz2_dgemm_ex")


def oz2_dsyrk(uplo, trans, n, k, alpha, A_ptr, lda, beta, C_ptr, ldc, num_moduli, stream=None):
    _check(lib().oz2_dsyrk(uplo.encode(), trans.encode(), n, k, float(alpha), A_ptr, lda, float(beta), C_ptr, ldc,
                           num_moduli, _stream_ptr(stream)), "oz2_dsyrk")


def oz2_dtrmm(side, uplo, transa, diag, m, n, alpha, A_ptr, lda, B_ptr, ldb, num_moduli, stream=None):
    _check(lib().oz2_dtrmm(side.encode(), uplo.encode(), transa.encode(), diag.encode(), m, n, float(alpha), A_ptr, lda,
                           B_ptr, ldb, num_moduli, _stream_ptr(stream)), "oz2_dtrmm")


def oz2_stage1_convert(m, n, k, A_ptr, lda, B_ptr, ldb, num_moduli, stream=None):
    _check(lib().oz2_stage1_convert(m, n, k, A_ptr, lda, B_ptr, ldb, num_moduli, _stream_ptr(stream)),
           "oz2_stage1_convert")


def oz2_stage2_gemm(m, n, k, num_moduli, stream=None):
    _check(lib().oz2_stage2_gemm(m, n, k, num_moduli, _stream_ptr(stream)), "oz2_stage2_gemm")


def oz2_stage3_crt(m, n, k, C_ptr, ldc, num_moduli, stream=None):
    _check(lib().oz2_stage3_crt(m, n, k, C_ptr, ldc, num_moduli, _stream_ptr(stream)), "oz2_stage3_crt")


def oz2_calibrate_mfma(workgroups, iters, random_operands, sink_ptr, clocks_ptr, stream=None):
    _check(lib().oz2_calibrate_mfma(workgroups, iters, int(random_operands), sink_ptr, clocks_ptr,
                                    _stream_ptr(stream)), "oz2_calibrate_mfma")


def host_kernel_choice(m, n, k, num_moduli, compute_units, call="dgemm"):
    """(vectors of the one-pass conversion, side of a thin product, edge of the product tiles) of a call."""
    out = (ctypes.c_int * 3)()
    _check(lib().oz2_host_kernel_choice(("dgemm", "dsyrk", "dtrmm").index(call), m, n, k, num_moduli, compute_units, out),
           "oz2_host_kernel_choice")
    return tuple(out)


def host_route(m, n, k, num_moduli, compute_units, call="dgemm", ta="N", tb="N"):
    """(operands in one pass, residues through the caches, edge of the bound tiles, kernel of lines 8-11) of a call."""
    out = (ctypes.c_int * 4)()
    _check(lib().oz2_host_route(("dgemm", "dsyrk", "dtrmm").index(call), ta.encode(), tb.encode(), m, n, k, num_moduli, compute_units, out),
           "oz2_host_route")
    return tuple(out)


def host_crt_element(num_moduli, cprod):
    arr = (ctypes.c_int32 * num_moduli)(*[int(c) for c in cprod])
    out = ctypes.c_double(0.0)
    _check(lib().oz2_host_crt_element(num_moduli, arr, ctypes.byref(out)), "oz2_host_crt_element")
    return out.value


def host_crt_element_digits(num_moduli, residues):
    arr = (ctypes.c_uint8 * num_moduli)(*[int(c) for c in residues])
    out = ctypes.c_double(0.0)
    name = "oz2_host_crt_element_wide_digits" if num_moduli > 16 else "oz2_host_crt_element_digits"
    _check(getattr(lib(), name)(num_moduli, arr, ctypes.byref(out)), name)
    return out.value


def host_residues(num_moduli, kappa, a, shift):
    out = (ctypes.c_int8 * num_moduli)()
    _check(lib().oz2_host_residues(num_moduli, kappa, float(a), int(shift), out), "oz2_host_residues")
    return list(out)


def host_product_residues(index, products, short=False):
    """products: contiguous int32 numpy array -> uint8 array of the same shape; short: as for inner dimensions up to 1024"""
    import numpy as np
    assert products.dtype == np.int32 and products.flags.c_contiguous
    out = np.empty(products.shape, dtype=np.uint8)
    name = "oz2_host_short_product_residues" if short else "oz2_host_product_residues"
    _check(getattr(lib(), name)(index, products.size, products.ctypes.data, out.ctypes.data), name)
    return out


OZ2_OPT_SHIFT_MODE, OZ2_OPT_PRODUCT_FORMAT, OZ2_OPT_GEMM_ALGORITHM, OZ2_OPT_KBLOCK, OZ2_OPT_BIT_SPLIT, OZ2_OPT_NONFINITE_CHECK = range(6)


class Context:
    """oz2_context: settings, workspace registration and lock of its own (see include/oz2.h).  The device buffer
    is torch's; the object keeps it alive as long as the context points at it."""

    def __init__(self):
        self.handle = ctypes.c_void_p()
        _check(lib().oz2_context_create(ctypes.byref(self.handle)), "oz2_context_create")
        self.buf = None

    def set(self, option, value):
        _check(lib().oz2_context_set(self.handle, int(option), int(value)), "oz2_context_set")

    def get(self, option):
        v = ctypes.c_int64(0)
        _check(lib().oz2_context_get(self.handle, int(option), ctypes.byref(v)), "oz2_context_get")
        return v.value

    def workspace_bytes(self, m, n, k, num_moduli):
        return int(lib().oz2_context_workspace_bytes(self.handle, m, n, k, num_moduli))

    def allocate_workspace(self, m, n, k, num_moduli, device="cuda:0"):
        import torch
        nbytes = self.workspace_bytes(m, n, k, num_moduli)
        if nbytes == 0:
            raise Oz2Error("invalid problem for a workspace")
        self.buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        off = (-self.buf.data_ptr()) % 256
        _check(lib().oz2_context_set_workspace(self.handle, self.buf.data_ptr() + off, nbytes), "oz2_context_set_workspace")
        return nbytes

    def dgemm(self, transa, transb, m, n, k, alpha, A_ptr, lda, B_ptr, ldb, beta, C_ptr, ldc, num_moduli, stream=None):
        _check(lib().oz2_context_dgemm(self.handle, transa.encode(), transb.encode(), m, n, k, float(alpha), A_ptr, lda,
                                       B_ptr, ldb, float(beta), C_ptr, ldc, num_moduli, _stream_ptr(stream)),
               "oz2_context_dgemm")

    def dsyrk(self, uplo, trans, n, k, alpha, A_ptr, lda, beta, C_ptr, ldc, num_moduli, stream=None):
        _check(lib().oz2_context_dsyrk(self.handle, uplo.encode(), trans.encode(), n, k, float(alpha), A_ptr, lda,
                                       float(beta), C_ptr, ldc, num_moduli, _stream_ptr(stream)), "oz2_context_dsyrk")

    def dtrmm(self, side, uplo, transa, diag, m, n, alpha, A_ptr, lda, B_ptr, ldb, num_moduli, stream=None):
        _check(lib().oz2_context_dtrmm(self.handle, side.encode(), uplo.encode(), transa.encode(), diag.encode(), m, n,
                                       float(alpha), A_ptr, lda, B_ptr, ldb, num_moduli, _stream_ptr(stream)),
               "oz2_context_dtrmm")

    def allocate_moe_workspace(self, layer, tokens, device="cuda:0"):
        """A workspace for w4_moe with up to that many tokens; any other that the context had is let go."""
        import torch
        nbytes = int(lib().oz2_w4_moe_workspace_bytes(layer.ref, tokens))
        if nbytes == 0:
            raise Oz2Error("invalid layer or number of tokens")
        buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        off = (-buf.data_ptr()) % 256
        _check(lib().oz2_context_set_workspace(self.handle, buf.data_ptr() + off, nbytes), "oz2_context_set_workspace")
        self.buf = buf
        return nbytes

    def w4_moe(self, layer, x, active=None, out=None, ids=None, weights=None, stream=None):
        """(y, ids, weights) of a MoeLayer for x (tokens, d); see w4_moe."""
        return _w4_moe(lib().oz2_context_w4_moe, "oz2_context_w4_moe", (self.handle,), layer, x, active, out, ids, weights, stream)

    def allocate_kv4_workspace(self, cache, table, tokens=0, heads=0, weights=False, keep=None):
        """A workspace on the cache's device for kv4_attention with up to that many new tokens of that many query heads (0: none), with weights if they are wanted,
        and for kv4_evict with that `keep` (None: none), on a table of that shape; any other that the context had is let go."""
        import torch
        sequences, max_pages = table.shape
        nbytes = []
        if heads:
            nbytes.append(int(lib().oz2_kv4_attention_workspace_bytes(cache.ref, sequences, max_pages, tokens, heads, int(bool(weights)))))
        if keep is not None:
            nbytes.append(int(lib().oz2_kv4_evict_workspace_bytes(cache.ref, sequences, max_pages, keep)))
        if not nbytes or 0 in nbytes:
            raise Oz2Error("invalid cache, table, tokens, heads or keep")
        buf = torch.empty(max(nbytes) + 256, dtype=torch.uint8, device=cache.device)
        off = (-buf.data_ptr()) % 256
        _check(lib().oz2_context_set_workspace(self.handle, buf.data_ptr() + off, max(nbytes)), "oz2_context_set_workspace")
        self.buf = buf
        return max(nbytes)

    def kv4_attention(self, cache, q, cu, table, lengths, scale=None, weights=None, out=None, stream=None):
        """Attention of the new tokens q over the cache; see kv4_attention."""
        return _kv4_attention(lib().oz2_context_kv4_attention, "oz2_context_kv4_attention", (self.handle,), cache, q, cu, table, lengths, scale, weights, out, stream)

    def kv4_evict(self, cache, table, lengths, positions, weights, keep, recent=0, out=None, stream=None):
        """(lengths, positions, weights) after an eviction; see kv4_evict."""
        return _kv4_evict(lib().oz2_context_kv4_evict, "oz2_context_kv4_evict", (self.handle,), cache, table, lengths, positions, weights, keep, recent, out, stream)

    def close(self):
        if self.handle:
            lib().oz2_context_destroy(self.handle)
            self.handle = ctypes.c_void_p()
        self.buf = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Workspace:
    """A torch-owned device buffer registered with the library (device memory only; no arithmetic)."""

    def __init__(self, m, n, k, num_moduli, device="cuda:0", product_format=None):
        import torch
        self.nbytes = workspace_bytes(m, n, k, num_moduli, product_format)
        if self.nbytes == 0:
            raise Oz2Error("invalid problem for a workspace")
        # enough for the form of the products that the settings in force prefer
        self.nbytes = max(self.nbytes, workspace_bytes_preferred(m, n, k, num_moduli))
        self.buf = torch.empty(self.nbytes + 256, dtype=torch.uint8, device=device)
        base = self.buf.data_ptr()
        self.offset = (-base) % 256
        self.ptr = base + self.offset
        set_workspace(self.ptr, self.nbytes)

    def close(self):
        """Unregister the buffer if the library still points at it.  The library keeps a bare pointer: once this
        object is gone the memory returns to the allocator, and a later call must find no workspace (status
        OZ2_ERR_WORKSPACE) instead of writing into memory that belongs to another tensor."""
        if getattr(self, "ptr", None) is not None and _registered_ptr == self.ptr and _lib is not None:
            set_workspace(None, 0)
        self.ptr = None

    def __del__(self):
        try:
            self.close()
        except Exception:   # interpreter shutdown: nothing left to protect
            pass

    def view(self, off, count, dtype):
        """1-D torch view of `count` elements of `dtype` starting `off` bytes into the workspace."""
        import torch
        esz = torch.empty((), dtype=dtype).element_size()
        return self.buf[self.offset + off: self.offset + off + count * esz].view(dtype)


def dgemm(A, B, num_moduli, C=None, workspace=None):
    """C = A @ B for column-major float64 torch tensors on the GPU (A: m x k, B: k x n given as the
    transposes of contiguous tensors, i.e. A.t().is_contiguous()).  Thin convenience wrapper."""
    import torch
    m, k = A.shape
    k2, n = B.shape
    assert k == k2 and A.dtype == torch.float64 and B.dtype == torch.float64
    assert A.t().is_contiguous() and B.t().is_contiguous(), "pass column-major matrices"
    if C is None:
        C = torch.empty((n, m), dtype=torch.float64, device=A.device).t()
    if workspace is None:
        workspace = Workspace(m, n, k, num_moduli, device=A.device)
    oz2_dgemm(m, n, k, A.data_ptr(), max(1, m), B.data_ptr(), max(1, k), C.data_ptr(), max(1, m), num_moduli)
    return C


OZ2_F32, OZ2_BF16, OZ2_F16 = range(3)
OZ2_SCORE_SOFTMAX, OZ2_SCORE_SIGMOID = range(2)
OZ2_ACT_SILU, OZ2_ACT_GELU = range(2)


class _W4(ctypes.Structure):
    _fields_ = ([(f, ctypes.c_int64) for f in ("n", "k", "group")] + [("codes", ctypes.c_void_p), ("ld_codes", ctypes.c_int64),
                ("scales", ctypes.c_void_p), ("ld_scales", ctypes.c_int64), ("zeros", ctypes.c_void_p), ("ld_zeros", ctypes.c_int64)] +
                [(f, ctypes.c_int64) for f in ("count", "stride_codes", "stride_scales", "stride_zeros")] + [("scale_type", ctypes.c_int)])


class _Moe(ctypes.Structure):
    _fields_ = ([(f, _W4) for f in ("gate", "up", "down")] + [("router", ctypes.c_void_p), ("ld_router", ctypes.c_int64), ("bias", ctypes.c_void_p)] +
                [(f, ctypes.c_int) for f in ("router_type", "top_k", "score", "renormalize", "activation")] + [("factor", ctypes.c_float)])


_types = {}
_dtypes = []


def _type_table():
    import torch
    _dtypes[:] = [torch.int32, torch.float32]
    _types.update({torch.float32: OZ2_F32, torch.bfloat16: OZ2_BF16, torch.float16: OZ2_F16})


def _type(dtype):
    if not _types:
        _type_table()
    if dtype not in _types:
        raise Oz2Error("float32, bfloat16 or float16 wanted, got %s" % dtype)
    return _types[dtype]


def _on_device(device, **tensors):
    if device.type != "cuda":
        raise Oz2Error("tensors on the GPU wanted, got %s" % device)
    for name, v in tensors.items():
        if v is not None and v.device != device:
            raise Oz2Error("%s is on %s, not on %s" % (name, v.device, device))


class W4Matrix:
    """A matrix held in 4 bits, or a stack of them (include/oz2.h): codes (.., n, bytes) uint8 with two codes to a byte, scales (.., n, groups)
    in float32, bfloat16 or float16, zeros (.., n, groups) uint8 or None.  The last dimension of each is without gaps; the object
    keeps the tensors."""

    def __init__(self, codes, scales, zeros=None, k=None, group=128):
        import torch
        parts = [codes, scales] + ([] if zeros is None else [zeros])
        if codes.dtype != torch.uint8 or (zeros is not None and zeros.dtype != torch.uint8):
            raise Oz2Error("codes and zeros are uint8")
        if codes.dim() not in (2, 3) or any(v.dim() != codes.dim() or v.shape[:-1] != codes.shape[:-1] for v in parts):
            raise Oz2Error("codes, scales and zeros are (n, .) or (count, n, .) alike")
        if any(v.shape[-1] > 1 and v.stride(-1) != 1 for v in parts):
            raise Oz2Error("the last dimension of codes, scales and zeros is contiguous")
        k = 2 * codes.shape[-1] if k is None else int(k)
        if group < 1 or k < 0 or codes.shape[-1] < (k + 1) // 2 or any(v.shape[-1] < -(-k // group) for v in parts[1:]):
            raise Oz2Error("codes, scales or zeros have too few columns for k = %d, group = %d" % (k, group))
        if any(v.device != codes.device for v in parts):
            raise Oz2Error("codes, scales and zeros are on different devices")
        self.codes, self.scales, self.zeros = codes, scales, zeros
        self.n, self.k, self.count, self.device = codes.shape[-2], k, codes.shape[0] if codes.dim() == 3 else 1, codes.device
        over = [v.stride(0) if v.dim() == 3 else 0 for v in parts] + [0]
        self.struct = _W4(self.n, k, group, codes.data_ptr(), codes.stride(-2), scales.data_ptr(), scales.stride(-2),
                          None if zeros is None else zeros.data_ptr(), 0 if zeros is None else zeros.stride(-2), self.count, *over[:3],
                          _type(scales.dtype))
        self.ref, self.index = ctypes.addressof(self.struct), codes.get_device()


def _rows(name, x, width):
    """leading dimension of a two-dimensional tensor with rows of that width, which are contiguous and do not overlap (an expanded one's do)"""
    shape, strides = x.shape, x.stride()  # (whole: each single one asked for costs as much)
    if len(shape) != 2 or shape[1] != width or (width > 1 and strides[1] != 1 and shape[0]):  # (strides of no rows say nothing)
        raise Oz2Error("%s is two-dimensional with contiguous rows of %d, got shape %s" % (name, width, tuple(shape)))
    pitch = strides[0]
    if pitch >= width:
        return pitch
    if shape[0] > 1:
        raise Oz2Error("the rows of %s overlap: %d wide, %d apart (an expanded tensor: pass a copy)" % (name, width, pitch))
    return width  # (of one row, or none)


def _refuse_gradient():
    import torch
    if torch.is_grad_enabled():
        raise Oz2Error("a tensor requires a gradient, which these products do not form: call them under torch.no_grad(), or with detached tensors")


_forward = None  # torch.autograd.forward_ad, whose _current_level is -1 where no tensor has a tangent


def _refuse_tangents(*tensors):
    """Tensors with a tangent require no gradient, and their tangents would be lost.  Called first of all, and inside a level of forward-mode
    differentiation."""
    global _forward
    if _forward is None:
        import torch.autograd.forward_ad as _forward
    if any(v is not None and _forward.unpack_dual(v).tangent is not None for v in tensors):
        raise Oz2Error("a tensor has a tangent, which these products do not form: call them with the primal of it")


_raw_stream = _current_device = None


def _stream_on(stream, index):
    """The stream's pointer; without one, that of the current stream of the device, which has to be the current one: kernels are launched there.
    A call of a few microseconds notices how long this takes: torch.cuda.current_stream() 2.7 us, torch's own accessor of the pointer 0.1."""
    global _raw_stream, _current_device
    if _current_device is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda i: torch.cuda.current_stream(i).cuda_stream)
        _current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    if _current_device() != index:
        raise Oz2Error("the tensors are on cuda:%d, the current device is cuda:%d" % (index, _current_device()))
    return _raw_stream(index) if stream is None else getattr(stream, "cuda_stream", stream)


def _new(x, shape, dtype, stream):
    """A tensor for results of a call on that stream (None: the current one).  It belongs to it: memory that the current stream has given back may still
    be written by what is pending there."""
    if stream is None or x.get_device() < 0:
        return x.new_empty(shape, dtype=dtype)
    import torch
    if not hasattr(stream, "cuda_stream"):
        pointer = getattr(stream, "value", stream)
        stream = torch.cuda.ExternalStream(pointer, device=x.device) if pointer else torch.cuda.default_stream(x.device)
    with torch.cuda.stream(stream):
        return x.new_empty(shape, dtype=dtype)


def w4_matvec(W, x, alpha=1.0, beta=0.0, c=None, out=None, stream=None):
    """alpha W x + beta c for every row of x (tokens, k), as (tokens, n) in the type of `out`, or of x where it is None; c is like the result.
    A result that is made here belongs to the stream of the call.  There is no gradient: tensors that require one are refused where one would be recorded, and those with a
    tangent everywhere."""
    if x.requires_grad or W.scales.requires_grad or (c is not None and c.requires_grad) or (out is not None and out.requires_grad):
        _refuse_gradient()
    if _forward is None or _forward._current_level >= 0:
        _refuse_tangents(x, W.scales, c, out)
    if out is None:
        out = _new(x, (x.shape[0], W.n), x.dtype, stream)
    index = x.get_device()
    if index < 0 or index != W.index or out.get_device() != index:
        _on_device(W.device, x=x, out=out)
    ldx, ldy, t = _rows("x", x, W.k), _rows("out", out, W.n), x.size(0)
    if out.size(0) != t:
        raise Oz2Error("x and out have the same number of tokens")
    if W.count != 1:
        raise Oz2Error("one matrix wanted, not a stack")
    c_ptr, ldc, y_type = None, 0, _type(out.dtype)
    if c is not None:
        _on_device(W.device, c=c)
        if c.dtype != out.dtype or c.size(0) != t:
            raise Oz2Error("c has the type and the number of tokens of the result")
        c_ptr, ldc = c.data_ptr(), _rows("c", c, W.n)
    rc = lib().oz2_w4_matvec(W.ref, t, alpha, _type(x.dtype), x.data_ptr(), ldx, beta, c_ptr, ldc, y_type, out.data_ptr(), ldy,
                             _stream_on(stream, index))
    if rc:
        _check(rc, "oz2_w4_matvec")
    return out


class MoeLayer:
    """A layer of gated experts on stacks of W4Matrix (include/oz2.h): router (experts, d), gate and up f x d, down d x f, bias (experts,)
    float32 or None.  The object keeps the tensors."""

    def __init__(self, router, gate, up, down, top_k, bias=None, score="softmax", renormalize=True, factor=1.0, activation="silu"):
        import torch
        if router.dim() != 2 or router.shape != (gate.count, gate.k) or (gate.k > 1 and router.stride(1) != 1):
            raise Oz2Error("router is (experts, d) = (%d, %d) with contiguous rows" % (gate.count, gate.k))
        ld_router = _rows("router", router, gate.k)
        if (up.n, up.k, up.count) != (gate.n, gate.k, gate.count) or (down.n, down.k, down.count) != (gate.k, gate.n, gate.count):
            raise Oz2Error("gate and up are f x d, down is d x f, each for every expert")
        if bias is not None and (bias.dtype != torch.float32 or tuple(bias.shape) != (gate.count,) or not bias.is_contiguous()):
            raise Oz2Error("bias is (experts,) in float32")
        if any(v.device != gate.device for v in (router, up, down) + (() if bias is None else (bias,))):
            raise Oz2Error("the parts of the layer are on different devices")
        self.router, self.gate, self.up, self.down, self.bias = router, gate, up, down, bias
        self.with_gradient = tuple(v for v in (router, bias, gate.scales, up.scales, down.scales) if v is not None)
        self.d, self.top_k, self.device = gate.k, int(top_k), gate.device
        self.struct = _Moe(gate.struct, up.struct, down.struct, router.data_ptr(), ld_router, None if bias is None else bias.data_ptr(),
                           _type(router.dtype), self.top_k, ("softmax", "sigmoid").index(score), int(bool(renormalize)),
                           ("silu", "gelu").index(activation), float(factor))
        self.ref = ctypes.addressof(self.struct)


def _w4_moe(call, name, first, layer, x, active, out, ids, weights, stream):
    import torch
    t, index = x.shape[0], x.get_device()
    if any(v is not None and v.requires_grad for v in (x, out, weights, *layer.with_gradient)):
        _refuse_gradient()
    if _forward is None or _forward._current_level >= 0:
        _refuse_tangents(x, out, weights, *layer.with_gradient)
    if out is None:
        out = _new(x, (t, layer.d), x.dtype, stream)
    if ids is None:
        ids = _new(x, (t, layer.top_k), torch.int32, stream)
    if weights is None:
        weights = _new(x, (t, layer.top_k), torch.float32, stream)
    if index < 0 or any(v.get_device() != index for v in (layer.router, out, ids, weights)):
        _on_device(layer.device, x=x, out=out, ids=ids, weights=weights)
    ldx, ldy = _rows("x", x, layer.d), _rows("out", out, layer.d)
    if out.size(0) != t:
        raise Oz2Error("x and out have the same number of tokens")
    for what, v, dtype in (("ids", ids, torch.int32), ("weights", weights, torch.float32)):
        if v.dtype != dtype or v.shape != (t, layer.top_k) or not v.is_contiguous():
            raise Oz2Error("%s is (tokens, top_k), %s, without gaps" % (what, dtype))
    mask = None
    if active is not None:
        _on_device(layer.device, active=active)
        if active.dtype not in (torch.bool, torch.uint8) or active.shape != (t,) or not active.is_contiguous():
            raise Oz2Error("active is (tokens,), bool or uint8")
        mask = active.data_ptr()
    rc = call(*first, layer.ref, t, _type(x.dtype), x.data_ptr(), ldx, mask, _type(out.dtype), out.data_ptr(), ldy, ids.data_ptr(), weights.data_ptr(),
              _stream_on(stream, index))
    if rc:
        _check(rc, name)
    return out, ids, weights


def w4_moe(layer, x, active=None, out=None, ids=None, weights=None, stream=None):
    """(y, ids, weights) of a MoeLayer for x (tokens, d), in the workspace that set_workspace registered; tokens whose `active` is 0 get 0.
    Streams and gradients as for w4_matvec."""
    return _w4_moe(lib().oz2_w4_moe, "oz2_w4_moe", (), layer, x, active, out, ids, weights, stream)


def w4_moe_workspace_bytes(layer, tokens):
    """Bytes that w4_moe takes of the registered workspace; 0 for an invalid layer or number of tokens."""
    return int(lib().oz2_w4_moe_workspace_bytes(layer.ref, tokens))


class _Kv4(ctypes.Structure):
    _fields_ = ([(f, ctypes.c_int64) for f in ("pages", "page_size", "heads", "dim")] + [(f, ctypes.c_void_p) for f in ("k_codes", "v_codes")] +
                [(f, ctypes.c_int64) for f in ("codes_page", "codes_head")] + [(f, ctypes.c_void_p) for f in ("k_scales", "v_scales")] +
                [(f, ctypes.c_int64) for f in ("scales_page", "scales_head")])


# oz2_rows, oz2_kv4_sequences and oz2_kv4_kept as bytes: objects of ctypes structures take several times as long to make
_pack_rows, _pack_sequences, _pack_kept = (struct.Struct(f).pack for f in ("Pqqi4x", "qqPqPqPPqqPqq", "PPqqPqq"))


def _heads(name, x, index, shape):
    """(tokens, heads, dim) tensor of that shape on device `index`, its last dimension contiguous, as the library sees it"""
    strides = x.stride()
    if x.shape != shape or len(strides) != 3 or (strides[2] != 1 and shape[2] > 1 and shape[0]):
        raise Oz2Error("%s is (tokens, heads, dim) = %s with the last dimension contiguous, got shape %s" % (name, tuple(shape), tuple(x.shape)))
    if x.get_device() != index or index < 0:
        raise Oz2Error("%s is on %s: tensors of one call are on one GPU" % (name, x.device))
    return _pack_rows(x.data_ptr(), strides[0], strides[1], _type(x.dtype))


def _integers(name, x, index, shape):
    if x.dtype is not _int32() or x.shape != shape or (x.stride()[-1] != 1 and shape[-1] > 1 and x.numel()):
        raise Oz2Error("%s is int32 of shape %s, its last dimension contiguous, got %s %s" % (name, tuple(shape), x.dtype, tuple(x.shape)))
    if x.get_device() != index:
        raise Oz2Error("%s is on %s: tensors of one call are on one GPU" % (name, x.device))
    return x.data_ptr()


def _int32():
    if not _types:
        _type_table()
    return _dtypes[0]


def _refuse_gradients(*tensors):
    for v in tensors:
        if v is not None and v.requires_grad:
            _refuse_gradient()
    if _forward is None or _forward._current_level >= 0:
        _refuse_tangents(*tensors)


def attention(q, k, v, cu, causal=True, scale=None, out=None, stream=None):
    """softmax(scale q k) v over packed prompts (include/oz2.h): q (tokens, heads, dim), k and v (tokens, kv_heads, dim) of one type in float32, bfloat16 or float16, cu
    (sequences + 1) int32 with the first row of every sequence; scale 1 / sqrt(dim) if None.  The result is like `out`, or q where it is None, and belongs to
    the stream of the call; rows behind the last sequence are left as they were (where the result is made here, they are not set).  There is no gradient:
    tensors that require one are refused where one would be recorded, and those with a tangent everywhere."""
    _refuse_gradients(q, k, v, out)
    index, shape, of_kv = q.get_device(), q.shape, k.shape
    rows_q = _heads("q", q, index, shape)
    tokens, heads, dim = shape
    if len(of_kv) != 3 or of_kv[0] != tokens or of_kv[2] != dim:
        raise Oz2Error("k and v are (tokens, kv_heads, dim) = (%d, ., %d), got shape %s" % (tokens, dim, tuple(of_kv)))
    rows_k, rows_v = _heads("k", k, index, of_kv), _heads("v", v, index, of_kv)
    if out is None:
        out = _new(q, shape, q.dtype, stream)
    rows_out, of_cu = _heads("out", out, index, shape), cu.shape
    if len(of_cu) != 1 or not of_cu[0]:
        raise Oz2Error("cu is (sequences + 1,) int32")
    rc = lib().oz2_attention(tokens, of_cu[0] - 1, _integers("cu", cu, index, of_cu), heads, of_kv[1], dim, max(dim, 1) ** -0.5 if scale is None else scale,
                             bool(causal), rows_q, rows_k, rows_v, rows_out, _stream_on(stream, index))
    if rc:
        _check(rc, "oz2_attention")
    return out


class KV4Cache:
    """A paged cache of keys and values held in 4 bits (include/oz2.h): codes (pages, kv_heads, page_size, dim / 2) uint8 and scales (pages, kv_heads, page_size, 2)
    float16 of keys and of values, alike in strides, the last two dimensions without gaps.  The object keeps the tensors."""

    def __init__(self, k_codes, k_scales, v_codes, v_scales):
        import torch
        if any(v.dim() != 4 for v in (k_codes, k_scales, v_codes, v_scales)):
            raise Oz2Error("codes are (pages, kv_heads, page_size, dim / 2), scales (pages, kv_heads, page_size, 2)")
        pages, heads, page_size, half = k_codes.shape
        for name, v, dtype, last in (("k_codes", k_codes, torch.uint8, half), ("v_codes", v_codes, torch.uint8, half), ("k_scales", k_scales, torch.float16, 2),
                                     ("v_scales", v_scales, torch.float16, 2)):
            if v.dtype != dtype or v.shape != (pages, heads, page_size, last):
                raise Oz2Error("%s is %s of shape %s, got %s %s" % (name, dtype, (pages, heads, page_size, last), v.dtype, tuple(v.shape)))
            if (last > 1 and v.stride(3) != 1) or (page_size > 1 and v.stride(2) != last):
                raise Oz2Error("the last two dimensions of %s are without gaps" % name)
            if v.device != k_codes.device:
                raise Oz2Error("the parts of the cache are on different devices")
        for a, b in ((k_codes, v_codes), (k_scales, v_scales)):
            if any(a.shape[i] > 1 and a.stride(i) != b.stride(i) for i in (0, 1)):
                raise Oz2Error("keys and values have the same strides")
        if k_scales.stride(0) % 2 or k_scales.stride(1) % 2:
            raise Oz2Error("strides of scales are whole pairs")
        self.k_codes, self.k_scales, self.v_codes, self.v_scales = k_codes, k_scales, v_codes, v_scales
        self.pages, self.heads, self.page_size, self.dim = pages, heads, page_size, 2 * half
        self.device, self.index = k_codes.device, k_codes.get_device()
        self.struct = _Kv4(pages, page_size, heads, 2 * half, k_codes.data_ptr(), v_codes.data_ptr(), k_codes.stride(0), k_codes.stride(1), k_scales.data_ptr(),
                           v_scales.data_ptr(), k_scales.stride(0) // 2, k_scales.stride(1) // 2)
        self.ref = ctypes.addressof(self.struct)

    @classmethod
    def empty(cls, pages, kv_heads, page_size, dim, device="cuda:0"):
        """A cache of new tensors: its places hold zeros."""
        import torch
        make = lambda last, dtype: torch.zeros((pages, kv_heads, page_size, last), dtype=dtype, device=device)
        return cls(make(dim // 2, torch.uint8), make(2, torch.float16), make(dim // 2, torch.uint8), make(2, torch.float16))


def _places(name, x, cache, sequences, capacity, dtype):
    shape, strides = x.shape, x.stride()
    if x.dtype is not dtype or len(shape) != 3 or shape[0] != sequences or shape[1] != cache.heads or shape[2] < capacity or (strides[2] != 1 and shape[2] > 1 and sequences):
        raise Oz2Error("%s is %s of shape (sequences, kv_heads, places) = (%d, %d, at least %d), its last dimension contiguous, got %s %s" % (
            name, dtype, sequences, cache.heads, capacity, x.dtype, tuple(shape)))
    if x.get_device() != cache.index:
        raise Oz2Error("%s is on %s: tensors of one call are on one GPU" % (name, x.device))
    return x.data_ptr(), strides[0], strides[1]


_nowhere = (0, 0, 0)


def _sequences(cache, table, lengths, tokens=0, cu=None, positions=None, weights=None):
    index, shape = cache.index, table.shape
    if index < 0:
        raise Oz2Error("tensors on the GPU wanted, got %s" % cache.device)
    if len(shape) != 2:
        raise Oz2Error("table is (sequences, pages) int32")
    sequences, max_pages = shape
    capacity, int32 = max_pages * cache.page_size, _int32()
    of_positions = _nowhere if positions is None else _places("positions", positions, cache, sequences, capacity, int32)
    of_weights = _nowhere if weights is None else _places("weights", weights, cache, sequences, capacity, _dtypes[1])
    return _pack_sequences(sequences, max_pages, _integers("table", table, index, shape), table.stride()[0], _integers("lengths", lengths, index, (sequences,)),
                           tokens, 0 if cu is None else _integers("cu", cu, index, (sequences + 1,)), *of_positions, *of_weights)


def kv4_append(cache, k, v, cu, table, lengths, at=None, positions=None, weights=None, held=None, stream=None):
    """Appends the new tokens k and v (tokens, kv_heads, dim), packed by cu (sequences + 1) int32, to their sequences' last places (include/oz2.h): table (sequences, pages)
    int32, lengths (sequences) int32 with the new tokens counted.  at (tokens) int32: positions of the new tokens, stored in positions (sequences, kv_heads,
    places) int32; weights, of that shape in float32: set to 0 in the new places; held: (k, v) like the arguments, for what the cache then holds of them."""
    held_k, held_v = _none if held is None else held
    _refuse_gradients(k, v, weights, held_k, held_v, cache.k_scales, cache.v_scales)
    index, shape = cache.index, k.shape
    if len(shape) != 3 or shape[1] != cache.heads or shape[2] != cache.dim:
        raise Oz2Error("k and v are (tokens, kv_heads, dim) = (., %d, %d), got shape %s" % (cache.heads, cache.dim, tuple(shape)))
    rows_k, rows_v, tokens = _heads("k", k, index, shape), _heads("v", v, index, shape), shape[0]
    on = _sequences(cache, table, lengths, tokens, cu, positions, weights)
    if (at is None) != (positions is None):
        raise Oz2Error("at and positions go together")
    rc = lib().oz2_kv4_append(cache.ref, on, None if at is None else _integers("at", at, index, (tokens,)), rows_k, rows_v,
                              None if held_k is None else _heads("held k", held_k, index, shape), None if held_v is None else _heads("held v", held_v, index, shape),
                              _stream_on(stream, index))
    if rc:
        _check(rc, "oz2_kv4_append")


_none = (None, None)


def _kv4_attention(call, name, first, cache, q, cu, table, lengths, scale, weights, out, stream):
    _refuse_gradients(q, weights, out, cache.k_scales, cache.v_scales)
    index, shape = cache.index, q.shape
    if len(shape) != 3 or shape[2] != cache.dim:
        raise Oz2Error("q is (tokens, heads, dim) = (., ., %d), got shape %s" % (cache.dim, tuple(shape)))
    rows_q = _heads("q", q, index, shape)
    if out is None:
        out = _new(q, shape, q.dtype, stream)
    rows_out = _heads("out", out, index, shape)
    on = _sequences(cache, table, lengths, shape[0], cu, None, weights)
    rc = call(*first, cache.ref, on, shape[1], shape[2] ** -0.5 if scale is None else scale, rows_q, rows_out, _stream_on(stream, index))
    if rc:
        _check(rc, name)
    return out


def kv4_attention(cache, q, cu, table, lengths, scale=None, weights=None, out=None, stream=None):
    """Attention of the new tokens q (tokens, heads, dim), packed by cu, over their sequences' places (include/oz2.h), in the workspace that set_workspace registered: a
    sequence's new tokens are its last ones, and each sees the places up to its own.  weights (sequences, kv_heads, places) float32: what every place received is
    added.  Streams, results and gradients as for attention."""
    return _kv4_attention(lib().oz2_kv4_attention, "oz2_kv4_attention", (), cache, q, cu, table, lengths, scale, weights, out, stream)


def kv4_attention_workspace_bytes(cache, table, tokens, heads, weights=False):
    """Bytes that kv4_attention takes of the registered workspace on a table of that shape; 0 for what is not valid."""
    return int(lib().oz2_kv4_attention_workspace_bytes(cache.ref, table.shape[0], table.shape[1], tokens, heads, int(bool(weights))))


def _kv4_evict(call, name, first, cache, table, lengths, positions, weights, keep, recent, out, stream):
    _refuse_gradients(weights, cache.k_scales, cache.v_scales, *(out or ()))
    if positions is None or weights is None:
        raise Oz2Error("positions and weights are needed")
    on = _sequences(cache, table, lengths, 0, None, positions, weights)
    kept = None
    if out is not None:
        to_lengths, to_positions, to_weights = out
        sequences, max_pages = table.shape
        capacity = max_pages * cache.page_size
        kept = _pack_kept(_integers("lengths", to_lengths, cache.index, (sequences,)), *_places("positions", to_positions, cache, sequences, capacity, _dtypes[0]),
                          *_places("weights", to_weights, cache, sequences, capacity, _dtypes[1]))
    rc = call(*first, cache.ref, on, keep, recent, kept, _stream_on(stream, cache.index))
    if rc:
        _check(rc, name)
    return (lengths, positions, weights) if out is None else tuple(out)


def kv4_evict(cache, table, lengths, positions, weights, keep, recent=0, out=None, stream=None):
    """(lengths, positions, weights) with at most `keep` places of every sequence (include/oz2.h): the `recent` newest stay, and of the others those with the largest
    weights; the cache's tokens move into the first `keep` places.  In place, or where out = (lengths, positions, weights) says; in the workspace that
    set_workspace registered."""
    return _kv4_evict(lib().oz2_kv4_evict, "oz2_kv4_evict", (), cache, table, lengths, positions, weights, keep, recent, out, stream)


def kv4_evict_workspace_bytes(cache, table, keep):
    """Bytes that kv4_evict takes of the registered workspace on a table of that shape; 0 for what is not valid."""
    return int(lib().oz2_kv4_evict_workspace_bytes(cache.ref, table.shape[0], table.shape[1], keep))
