"""The calls of csrc/fastcall.cpp through ctypes: the same functions with the same arguments, several microseconds a call slower,
for a package whose call layer has not been built (it needs torch's headers; the library itself does not)."""
from __future__ import annotations

import ctypes

import torch


class Calls:
    def __init__(self, lib, stream):
        """lib: the library, with its signatures set; stream: what turns a stream argument into a handle."""
        self.lib, self.handle = lib, stream

    def _matrix(self, t):
        if t is None:
            return None, 0
        if not isinstance(t, torch.Tensor):
            raise TypeError("expected a tensor")
        assert t.dim() == 2 and t.stride(1) == 1 and t.dtype == torch.float32, "expected a float32 matrix with contiguous rows"
        return t.data_ptr(), t.stride(0)

    def _memory(self, t):
        return t if t is None or isinstance(t, int) else t.data_ptr()

    def _matrix_with_ld(self, t, ld):
        return self._matrix(t) if ld is None else (self._memory(t), ld)

    def forward(self, layer, X, Y, batch, stream):
        return self.lib.sparse_linear_forward(layer, *self._matrix(X), *self._matrix(Y), batch, self.handle(stream))

    def backward(self, layer, X, Y, dY, dX, dvalues, dbias, batch, stream):
        return self.lib.sparse_linear_backward(layer, *self._matrix(X), *self._matrix(Y), *self._matrix(dY), *self._matrix(dX), self._memory(dvalues),
                                               self._memory(dbias), batch, self.handle(stream))

    def update(self, values, velocity, grad, n, lr, momentum, nesterov, stream):
        step = self.lib.sgd_update_values_nesterov if nesterov else self.lib.sgd_update_values
        return step(self._memory(values), self._memory(velocity), self._memory(grad), n, lr, momentum, self.handle(stream))

    def train_step(self, mlp, X, ldx, labels, batch, lr, momentum, workspace, loss, stream):
        return self.lib.mlp_train_step(mlp, *self._matrix_with_ld(X, ldx), self._memory(labels), batch, lr, momentum, workspace.data_ptr(), workspace.nbytes,
                                       self._memory(loss), self.handle(stream))

    def mlp_forward(self, mlp, X, ldx, batch, workspace, stream):
        return self.lib.mlp_forward(mlp, *self._matrix_with_ld(X, ldx), batch, workspace.data_ptr(), workspace.nbytes, self.handle(stream))

    def view(self, workspace, rows, batch, ld, offset):
        return workspace.as_strided((rows, batch), (ld, 1), workspace.storage_offset() + offset)

    # ---- mixtures and clipped gradients: with the looks at types, shapes and devices of csrc/fastcall.cpp

    def _numbers(self, *numbers):
        """ctypes would cut them."""
        for n in numbers:
            if not -2 ** 31 <= n < 2 ** 31:
                raise OverflowError(f"{n} does not fit 32 bits")

    def _tensor(self, t, name, dtype):
        if not isinstance(t, torch.Tensor):
            raise TypeError("expected a tensor")
        assert t.dtype == dtype, f"{name}: {'float32' if dtype == torch.float32 else dtype} expected"
        assert t.is_cuda, f"{name}: a tensor on the GPU expected"
        assert t.get_device() == torch.cuda.current_device(), f"{name}: a tensor on the current device expected"
        return t

    def _sized(self, t, name, rows, columns, dtype=torch.float32, optional=False):
        if optional and t is None:
            return None, 0
        t = self._tensor(t, name, dtype)
        assert t.dim() == 2 and t.stride(1) == 1 and t.size(0) >= rows and t.size(1) >= columns, f"{name}: a matrix of the call's sizes with contiguous rows expected"
        step = t.stride(0) if t.size(0) > 1 else t.size(1)
        assert step < 2 ** 31, f"{name}: rows less than 2^31 entries apart expected"
        return t.data_ptr(), step

    def _blocks(self, t, name, experts, features, capacity, optional=False):
        if optional and t is None:
            return None, 0
        t = self._tensor(t, name, torch.float32)
        assert t.dim() == 3 and t.stride(2) == 1 and t.size(0) >= experts and t.size(1) == features and t.size(2) >= capacity, \
            f"{name}: blocks (experts, features, capacity) with contiguous rows expected"
        step = t.stride(1) if features > 1 else t.stride(0) if t.size(0) > 1 else t.size(2)
        assert step < 2 ** 31 and (t.size(0) <= 1 or t.stride(0) == features * step), f"{name}: blocks right behind each other expected"
        return t.data_ptr(), step

    def _vector(self, t, name, n, dtype=torch.float32, optional=False):
        if optional and t is None:
            return None
        t = self._tensor(t, name, dtype)
        assert t.numel() >= n and t.is_contiguous(), f"{name}: a contiguous array of the call's size expected"
        return t.data_ptr()

    def _scratch(self, t, name):
        if t is None:
            return None, 0
        if not isinstance(t, torch.Tensor):
            raise TypeError("expected a tensor")
        t = self._tensor(t, name, t.dtype)
        assert t.is_contiguous(), f"{name}: contiguous memory expected"
        return t.data_ptr(), t.nbytes

    def _arrays(self, ts, name, counts=None):
        assert isinstance(ts, (list, tuple)), f"{name}: a list of tensors expected"
        assert counts is None or len(ts) == len(counts), f"{name}: as many tensors as gradients expected"
        for t in ts:
            assert self._tensor(t, name, torch.float32).is_contiguous(), f"{name}: contiguous arrays expected"
        lengths = [t.numel() for t in ts]
        assert counts is None or lengths == counts, f"{name}: arrays as long as the gradients expected"
        return (ctypes.c_void_p * len(ts))(*[t.data_ptr() for t in ts]), lengths

    def _same(self, name, of, k, *lds):
        assert k <= 1 or len(set(lds)) == 1, f"{name}: the row stride of {of} expected"

    def route(self, Z, bias, experts, batch, k, groups, top_groups, flags, scale, chosen, weights, stream):
        self._numbers(experts, batch, k, groups, top_groups, flags)
        z = self._sized(Z, "Z", experts, batch)
        b = self._vector(bias, "bias", experts, optional=True)
        c, ldk = self._sized(chosen, "chosen", k, batch, torch.int32)
        w, ldw = self._sized(weights, "weights", k, batch)
        self._same("weights", "chosen", k, ldk, ldw)
        return self.lib.expert_route(*z, b, experts, batch, k, groups, top_groups, flags, scale, c, w, ldk, self.handle(stream))

    def route_backward(self, Z, chosen, dweights, experts, batch, k, flags, scale, dZ, stream):
        self._numbers(experts, batch, k, flags)
        z = self._sized(Z, "Z", experts, batch)
        c, ldk = self._sized(chosen, "chosen", k, batch, torch.int32)
        w, ldw = self._sized(dweights, "dweights", k, batch)
        d = self._sized(dZ, "dZ", experts, batch)
        self._same("dweights", "chosen", k, ldk, ldw)
        return self.lib.expert_route_backward(*z, c, w, ldk, experts, batch, k, flags, scale, *d, self.handle(stream))

    def place(self, chosen, experts, batch, k, capacity, slots, counts, placement, stream):
        self._numbers(experts, batch, k, capacity)
        c, ldk = self._sized(chosen, "chosen", k, batch, torch.int32)
        s, lds = self._sized(slots, "slots", k, batch, torch.int32, True)
        n = self._vector(counts, "counts", experts, torch.int32, True)
        if s is not None:
            self._same("slots", "chosen", k, ldk, lds)
        return self.lib.expert_place(c, ldk, experts, batch, k, capacity, s, n, *self._scratch(placement, "placement"), self.handle(stream))

    def dispatch(self, X, placement, features, experts, batch, k, capacity, Xe, stream):
        self._numbers(features, experts, batch, k, capacity)
        x = self._sized(X, "X", features, batch)
        p = self._scratch(placement, "placement")
        xe = self._blocks(Xe, "Xe", experts, features, capacity)
        return self.lib.expert_dispatch(*x, *p, features, experts, batch, k, capacity, *xe, self.handle(stream))

    def combine(self, Ye, placement, weights, features, experts, batch, k, capacity, Y, stream):
        self._numbers(features, experts, batch, k, capacity)
        ye = self._blocks(Ye, "Ye", experts, features, capacity)
        p = self._scratch(placement, "placement")
        w = self._sized(weights, "weights", k, batch, optional=True)
        y = self._sized(Y, "Y", features, batch)
        return self.lib.expert_combine(*ye, *p, *w, features, experts, batch, k, capacity, *y, self.handle(stream))

    def combine_backward(self, Ye, dY, placement, weights, features, experts, batch, k, capacity, dYe, dweights, workspace, stream):
        self._numbers(features, experts, batch, k, capacity)
        ye, lde = self._blocks(Ye, "Ye", experts, features, capacity, True)
        dy = self._sized(dY, "dY", features, batch)
        p = self._scratch(placement, "placement")
        w, ldk = self._sized(weights, "weights", k, batch, optional=True)
        dye, ldd = self._blocks(dYe, "dYe", experts, features, capacity, True)
        dw, lddw = self._sized(dweights, "dweights", k, batch, optional=True)
        assert ye is None or dye is None or lde == ldd, "dYe: the row stride of Ye expected"
        if w is not None and dw is not None:
            self._same("dweights", "weights", k, ldk, lddw)
        return self.lib.expert_combine_backward(ye, lde if ye is not None else ldd, *dy, *p, w, ldk if w is not None else lddw, features, experts, batch, k, capacity,
                                                dye, dw, *self._scratch(workspace, "workspace"), self.handle(stream))

    def norm(self, grads, workspace, norm, stream):
        g, counts = self._arrays(grads, "grads")
        return self.lib.gradient_norm(len(counts), g, (ctypes.c_int64 * len(counts))(*counts), *self._scratch(workspace, "workspace"),
                                      self._vector(norm, "norm", 1, optional=True), self.handle(stream))

    def clip(self, grads, clipped, max_norm, workspace, norm, stream):
        g, counts = self._arrays(grads, "grads")
        c, _ = self._arrays(clipped, "clipped", counts)
        return self.lib.gradient_clip(len(counts), g, c, (ctypes.c_int64 * len(counts))(*counts), max_norm, *self._scratch(workspace, "workspace"),
                                      self._vector(norm, "norm", 1, optional=True), self.handle(stream))

    def update_clipped(self, values, velocities, grads, lr, momentum, max_norm, nesterov, workspace, norm, stream):
        g, counts = self._arrays(grads, "grads")
        w, _ = self._arrays(values, "values", counts)
        v, _ = self._arrays(velocities, "velocities", counts)
        return self.lib.sgd_update_clipped(len(counts), w, v, g, (ctypes.c_int64 * len(counts))(*counts), lr, momentum, max_norm, int(nesterov),
                                           *self._scratch(workspace, "workspace"), self._vector(norm, "norm", 1, optional=True), self.handle(stream))
