"""ctypes mirrors of the argument structures of include/qsr.h for layer norm, the embedding and the gated recurrence."""
import ctypes as C


def _struct(name, spec):
    kinds = {"i": C.c_int32, "l": C.c_int64, "p": C.c_void_p, "d": C.c_double}
    return type(name, (C.Structure,), {"_fields_": [(n, kinds[k]) for k, names in spec for n in names.split()]})


LayerNormArgs = _struct("LayerNormArgs", [
    ("i", "K type y_type"), ("l", "rows d"), ("p", "x residual weight bias sum y scale mean rstd"),
    ("l", "x_stride residual_stride sum_stride y_stride weight_stride bias_stride"), ("d", "eps")])
LayerNormBackwardArgs = _struct("LayerNormBackwardArgs", [
    ("i", "K type"), ("l", "rows d"), ("p", "y_grad sum weight mean rstd residual_grad x_grad weight_grad bias_grad"),
    ("l", "y_grad_stride sum_stride residual_grad_stride x_grad_stride weight_stride")])
EmbeddingArgs = _struct("EmbeddingArgs", [
    ("i", "K type y_type reserved"), ("l", "tokens_each vocab d"), ("p", "table tokens y"), ("l", "table_stride worker_stride y_stride"),
    ("d", "scale")])
EmbeddingBackwardArgs = _struct("EmbeddingBackwardArgs", [
    ("i", "K type grad_type accumulate"), ("l", "tokens_each vocab d"), ("p", "y_grad tokens grad"),
    ("l", "y_grad_stride grad_stride worker_stride"), ("d", "scale")])
GatedScanArgs = _struct("GatedScanArgs", [
    ("i", "type input"), ("l", "batch steps d"), ("p", "x gate initial reset lengths h last states"),
    ("l", "x_batch_stride x_stride gate_batch_stride gate_stride h_batch_stride h_stride")])
GatedScanBackwardArgs = _struct("GatedScanBackwardArgs", [
    ("i", "type input"), ("l", "batch steps d"), ("p", "h_grad x gate states last_grad reset lengths x_grad gate_grad initial_grad"),
    ("l", "h_grad_batch_stride h_grad_stride x_batch_stride x_stride gate_batch_stride gate_stride x_grad_batch_stride x_grad_stride "
          "gate_grad_batch_stride gate_grad_stride")])
